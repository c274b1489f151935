// Products of 8-bit floating-point codes (e4m3, e5m2) with a power-of-two scale for each block of 128 along the reduction:
//   out[m, n]   = sum_k a[m,k] sa[m, k/128] b[g][n,k] sb[g][n/128, k/128] + bias[g][n]        rows m of group g (forward)
//   out[m, n]   = sum_k a[m,k] sa[m, k/128] b[g][k,n] sb[g][k/128, n/128]                      the same weights read across (input gradient)
// The dense product is the grouped one with a single group.
//
// The tensor cores apply the scales themselves (tcgen05 kind::mxf8f6f4 with block scales: one byte for 32 elements, here the same
// byte for the four steps of a block), so partial sums never leave tensor memory before a tile is done.
//
// One persistent kernel.  The weights are the tile's 128 rows, the tokens its
// columns: their number is given to the instruction at run time, so a group of 37 rows costs 48 columns and not a tile.  Weights read
// across are taken as they lie in memory: the tensor core reads them MN-major.
// Warp 0 loads codes by TMA, warp 1 multiplies into one of two accumulators, warp 2 fetches the tensor maps, warp 3 works out the tiles,
// warps 4..11 store the previous one, warps 12..15 put the scales into tensor memory.  All waits are bounded.
//
// No access leaves the caller's buffers: tensor maps describe exactly these, so what lies outside is filled with zeros or not
// stored; offsets are held to 0..M before they are used, and a tile's rows end with its group; scales are read 16 bytes at a time from
// multiples of 16 inside a row.
//
// 10000 x 4096 x 4096, e4m3 to bf16: 117 us from cold, 2870 T operations/s; repeated it is held by the power limit, 145 us at 1335 MHz, 193000
// clocks (zeros in the place of the tokens: 101 us at 1878 MHz, 191000 clocks).  The tensor pipe is busy 70 % of the active clocks.
#pragma once
#include <cuda.h>
#include "qnn_f8.cuh"
#include "qnn_tc_ptx.cuh"

namespace qnn {

enum F8Mode { FORWARD = 0, ACROSS = 1 };

struct F8Params {
    int64_t M;                       // rows of a (tokens) of all groups; offsets are held to 0..M
    int32_t N;                       // channels: rows of the tile's operand
    int32_t nkb;                     // blocks of the reduction
    int32_t groups;
    const int64_t *offsets;          // [groups + 1] or NULL: one group of all rows
    const uint8_t *w_scale; int64_t ld_ws, stride_ws;      // scales of the tile's rows
    const uint8_t *x_scale; int64_t ld_xs;                 // scales of the tile's columns
    const float *bias;               // [groups, N] or NULL
    void *out; int64_t ldo;
    int32_t vec_out;                 // rows of the output may be written in 16-byte pieces
    int32_t has_maps;                // 0: an empty reduction, nothing is loaded
    int32_t tma_out;                 // whole blocks of the output leave as bulk stores
    int32_t tiles_c;                 // tiles of channels
    int32_t nt;                      // columns of a tile at most
    int32_t step;                    // ... a multiple of this many, but for the last ones
    int32_t acc1;                    // tensor-memory column of the second accumulator
    int32_t overlap;                 // 1: its first 32 columns are the first one's last
    int32_t chunks, chunk;           // chunks of tokens and tokens of each: one group of all rows (offsets NULL)
    int32_t super;                   // chunks of tokens that go through all channels before the next ones
    uint32_t idesc;                  // without N and the scales' byte
};

struct F8Call {
    const char *what;
    const void *w; int w_type; int64_t w_rows, w_cols, ld_w, stride_w;      // as they lie in memory, `groups` of them stride_w bytes apart
    int32_t w_count;
    const void *x; int x_type; int64_t x_rows, x_cols, ld_x;
};

// How a product runs: columns that the kernel's tile has room for, CTAs that share a tile (ctas: a pair, split: parts of the
// reduction), columns of the tiles of this product.
struct F8Choice {
    int width, ctas, split, nt;
};
constexpr int chunk_step(int width) { return width >= 64 ? 32 : 16; }      // (blocks of 32 columns leave as one store)

// (see qnn_gemm_f8.cu)
F8Choice choose_f8(int64_t M, int64_t groups, int64_t N, int64_t nkb, bool one_group);
int pairs_resident_f8();
// one translation unit each; the status word of its waits: reads and clears it
int run_f8_forward(const F8Call &c, const F8Params &p, int out_type, cudaStream_t st);
int run_f8_across(const F8Call &c, const F8Params &p, int out_type, cudaStream_t st);
int f8_forward_status(int *code);
int f8_across_status(int *code);

namespace {

constexpr int F8_THREADS = 512;
template <int NT, int MODE, int CTAS, typename TOUT, int SPLIT = 1>
struct F8Cfg {
    static constexpr int A_BYTES = BM * BKB;
    static constexpr int BROWS = NT / CTAS > 128 ? 256 : NT / CTAS > 64 ? 128 : NT / CTAS > 32 ? 64 : 32;   // rows (columns, MN-major) a CTA loads at most
    static constexpr int B_BYTES = BROWS * BKB;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr bool CUT = SPLIT > 1;
    // Up to 16 tokens: CTAs send their sums to the one that joins them (no cluster-wide barrier behind the products: 16 x 4096 x 4096
    // 8.3 -> 7.2 us), and two CTAs fit an SM: one's set-up and join overlap the other's stream of weights.
    static constexpr bool PUSH = CUT && NT == 16;
    static constexpr int RESIDENT = PUSH ? 2 : 1;
    static constexpr int JOIN_BYTES = PUSH ? NT * BM * 4 : 0;           // what the CTAs of a cluster send here
    static constexpr int STG_BYTES = CUT ? 1024 : 8 * 32 * 32 * (int)sizeof(TOUT);   // a block of 32 x 32 results for each storing warp
    static constexpr int SFB = (NT + 127) / 128;                        // pieces of 128 columns
    static constexpr int SF_COLS = 4 + 4 * SFB;                         // tensor-memory columns of one word's scales
    // Tensor memory: two accumulators and two words of scales.  With 256 columns each that is more than there is: the accumulators
    // then share 32 columns, which are drained first.
    static constexpr int SF_BASE = NT == 256 ? 512 - 2 * SF_COLS : 2 * NT;
    static constexpr int TMEM_NEED = SF_BASE + 2 * SF_COLS;
    static constexpr int TMEM = TMEM_NEED <= 64 ? 64 : TMEM_NEED <= 128 ? 128 : TMEM_NEED <= 256 ? 256 : 512;
    // Scales on their way: 16 blocks' bytes of every column, handed from warp to warp.
    static constexpr int Q_BYTES = (16 * NT + 127) / 128 * 128;
    static constexpr int QS = 2;
    static constexpr int TABLE_BYTES = CUT ? 0 : 2 * 4 * (MAX_GROUPS + 8);          // (reductions are cut for one group only)
    static constexpr int BAR_BYTES = 320;
    static constexpr int RING_BYTES = 64 * 32;                          // tiles on their way to the roles
    static constexpr int AUX = STG_BYTES + JOIN_BYTES + QS * Q_BYTES + RING_BYTES + TABLE_BYTES + BAR_BYTES + 1024;
    static constexpr int MAXS = ((RESIDENT == 2 ? 113 * 1024 : SMEM_LIMIT) - AUX) / STAGE_BYTES;
    static constexpr int STAGES = MAXS > 8 ? 8 : MAXS;
    static constexpr int STG_OFFSET = STAGES * STAGE_BYTES;
    static constexpr int JOIN_OFFSET = STG_OFFSET + STG_BYTES;
    static constexpr int Q_OFFSET = JOIN_OFFSET + JOIN_BYTES;
    static constexpr int RING_OFFSET = Q_OFFSET + QS * Q_BYTES;
    static constexpr int TABLE_OFFSET = RING_OFFSET + RING_BYTES;
    static constexpr int BAR_OFFSET = TABLE_OFFSET + TABLE_BYTES;
    static constexpr int TOTAL = BAR_OFFSET + BAR_BYTES + 1024;
    static_assert(TMEM_NEED <= 512 && (2 * STAGES + QS + 11) * 8 + 16 <= BAR_BYTES && RESIDENT * (TOTAL + 1024) <= 228 * 1024, "configuration");
    // The scales' warps learn from a stage's barrier that the word before the last one has been used: the products cannot be more than
    // four blocks past it by then, so the barrier must not come round within five.
    static_assert(STAGES >= 5, "configuration");
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
// One block of the reduction as ONE instruction stream: poll the NEXT stage's full barrier, issue the block's four steps of 32 (A_STEP
// and B_STEP apart in the descriptors' address field), commit them to this stage's empty barrier (a pair: of both CTAs), and only then
// read the poll's result, whose latency hides behind the issue.  Returns non-zero when the next stage has landed.
template <int CTAS, uint32_t A_STEP, uint32_t B_STEP>
__device__ __forceinline__ uint32_t umma_f8_block(uint32_t next_full_bar, uint32_t next_parity, uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi,
                                                  uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate, uint32_t sf, uint32_t empty_bar)
{
    uint32_t ready;
#define QNN_F8_BLOCK(GROUP, COMMIT)                                                                                                          \
    asm volatile("{\n"                                                                                                                      \
                 ".reg .pred P, Q, T;\n"                                                                                                    \
                 ".reg .b64 a0, a1, a2, a3, b0, b1, b2, b3;\n"                                                                              \
                 ".reg .b32 t1, t2, t3, u1, u2, u3, sb;\n"                                                                                  \
                 ".reg .b16 both;\n"                                                                                                        \
                 "mov.b16 both, 3;\n"                                                                                                       \
                 "mbarrier.test_wait.parity.shared::cta.b64 Q, [%1], %2;\n"                                                                  \
                 "setp.ne.b32 P, %9, 0;\n"                                                                                                  \
                 "setp.eq.b32 T, 0, 0;\n"                                                                                                   \
                 "add.u32 sb, %10, 4;\n"                                                                                                    \
                 "add.u32 t1, %4, %12;\n add.u32 t2, t1, %12;\n add.u32 t3, t2, %12;\n"                                                   \
                 "add.u32 u1, %6, %13;\n add.u32 u2, u1, %13;\n add.u32 u3, u2, %13;\n"                                                   \
                 "mov.b64 a0, {%4, %5};\n mov.b64 a1, {t1, %5};\n mov.b64 a2, {t2, %5};\n mov.b64 a3, {t3, %5};\n"                       \
                 "mov.b64 b0, {%6, %7};\n mov.b64 b1, {u1, %7};\n mov.b64 b2, {u2, %7};\n mov.b64 b3, {u3, %7};\n"                       \
                 "tcgen05.mma.cta_group::" GROUP ".kind::mxf8f6f4.block_scale.scale_vec::1X [%3], a0, b0, %8, [%10], [sb], P;\n"            \
                 "tcgen05.mma.cta_group::" GROUP ".kind::mxf8f6f4.block_scale.scale_vec::1X [%3], a1, b1, %8, [%10], [sb], T;\n"            \
                 "tcgen05.mma.cta_group::" GROUP ".kind::mxf8f6f4.block_scale.scale_vec::1X [%3], a2, b2, %8, [%10], [sb], T;\n"            \
                 "tcgen05.mma.cta_group::" GROUP ".kind::mxf8f6f4.block_scale.scale_vec::1X [%3], a3, b3, %8, [%10], [sb], T;\n"            \
                 "tcgen05.commit.cta_group::" GROUP ".mbarrier::arrive::one.shared::cluster" COMMIT ";\n"                                   \
                 "selp.u32 %0, 1, 0, Q;\n"                                                                                                  \
                 "}\n"                                                                                                                      \
                 : "=r"(ready)                                                                                                              \
                 : "r"(next_full_bar), "r"(next_parity), "r"(d_tmem), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate), \
                   "r"(sf), "r"(empty_bar), "n"(A_STEP), "n"(B_STEP)                                                                        \
                 : "memory")
    if (CTAS == 2) QNN_F8_BLOCK("2", ".multicast::cluster.b64 [%11], both");
    else QNN_F8_BLOCK("1", ".b64 [%11]");
#undef QNN_F8_BLOCK
    return ready;
}
// this warp's 32 lanes of four / eight tensor-memory columns
__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t *v)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
// for all lanes of a warp at once, which leave it together
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, int code)
{
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, code));
}
// (never suspends the thread, as a try_wait may)
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
template <int CTAS>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if (CTAS == 2) umma_commit_pair(bar);
    else umma_commit(bar);
}
// 32 lanes x 32 columns as fragments of 8 x 8: v[16 h + 4 c + 2 u + e] of lane 4 r + t is lane 16 h + 8 u + r, column 8 c + 2 t + e
__device__ __forceinline__ void tmem_ld_frag(uint32_t taddr, uint32_t (&v)[32])
{
#pragma unroll
    for (int h = 0; h < 2; ++h)
        asm volatile(
            "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
            "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
            : "=r"(v[16 * h]), "=r"(v[16 * h + 1]), "=r"(v[16 * h + 2]), "=r"(v[16 * h + 3]), "=r"(v[16 * h + 4]), "=r"(v[16 * h + 5]),
              "=r"(v[16 * h + 6]), "=r"(v[16 * h + 7]), "=r"(v[16 * h + 8]), "=r"(v[16 * h + 9]), "=r"(v[16 * h + 10]), "=r"(v[16 * h + 11]),
              "=r"(v[16 * h + 12]), "=r"(v[16 * h + 13]), "=r"(v[16 * h + 14]), "=r"(v[16 * h + 15])
            : "r"(taddr + ((uint32_t)(16 * h) << 16)) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// four 8 x 8 blocks of 16-bit elements, transposed: lane 8 m + j gives the address of row j (a column of the fragment) of block m
__device__ __forceinline__ void stmatrix_trans(uint32_t addr, const uint32_t (&o)[4])
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
}
// arrival on a barrier of the pair's leader (a shared::cluster address) or of this CTA
template <int CTAS>
__device__ __forceinline__ void arrive_at_leader(uint32_t bar)
{
    if (CTAS == 2) mbar_arrive_cluster(bar);
    else mbar_arrive(bar);
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
__device__ __forceinline__ float4 ld_peer_f32x4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
// asynchronous store of W words into another CTA's shared memory that reports its bytes to a barrier there
template <int W>
__device__ __forceinline__ void send(uint32_t addr, const uint32_t *v, uint32_t bar)
{
    if constexpr (W == 4)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                     ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(bar) : "memory");
    else
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(bar) : "memory");
}
// (volatile: issued where it stands, well before its use)
__device__ __forceinline__ uint4 ldg128(const uint8_t *ptr)
{
    uint4 v;
    asm volatile("ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(ptr));
    return v;
}
__device__ __forceinline__ void expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// One stage of the loading warp in the same way: poll the NEXT stage's empty barrier, announce this stage's bytes (a pair: those of both
// CTAs, by its leader), issue the load of the tile's rows and the first of its columns.
template <int CTAS>
__device__ __forceinline__ uint32_t tma_f8_stage(uint32_t next_empty_bar, uint32_t next_parity, uint32_t full_bar, uint32_t bytes, uint32_t announce,
                                                 uint32_t dst_a, const CUtensorMap *map_a, int32_t ax, int32_t ay, int32_t az, uint32_t dst_b,
                                                 const CUtensorMap *map_b, int32_t bx, int32_t by)
{
    uint32_t ready;
#define QNN_F8_STAGE(GROUP)                                                                                                                       \
    asm volatile("{\n"                                                                                                                          \
                 ".reg .pred Q, L;\n"                                                                                                           \
                 "mbarrier.test_wait.parity.shared::cta.b64 Q, [%1], %2;\n"                                                                      \
                 "setp.ne.b32 L, %14, 0;\n"                                                                                                     \
                 "@L mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%3], %4;\n"                                                              \
                 "cp.async.bulk.tensor.3d" GROUP ".shared::cluster.global.mbarrier::complete_tx::bytes [%5], [%6, {%7, %8, %9}], [%3];\n"       \
                 "cp.async.bulk.tensor.2d" GROUP ".shared::cluster.global.mbarrier::complete_tx::bytes [%10], [%11, {%12, %13}], [%3];\n"       \
                 "selp.u32 %0, 1, 0, Q;\n"                                                                                                      \
                 "}\n"                                                                                                                          \
                 : "=r"(ready)                                                                                                                  \
                 : "r"(next_empty_bar), "r"(next_parity), "r"(full_bar), "r"(bytes), "r"(dst_a), "l"(map_a), "r"(ax), "r"(ay), "r"(az),         \
                   "r"(dst_b), "l"(map_b), "r"(bx), "r"(by), "r"(announce)                                                                      \
                 : "memory")
    if (CTAS == 2) QNN_F8_STAGE(".cta_group::2");
    else QNN_F8_STAGE("");
#undef QNN_F8_STAGE
    return ready;
}

// ---- tiles -------------------------------------------------------------------------------------------------------

struct F8Tile {
    int32_t g;                       // group
    int32_t c0;                      // first channel (of the pair)
    int32_t m0;                      // first token
    int32_t cols;                    // columns with a result
    int32_t n;                       // columns multiplied: rounded up to what the instruction takes
    int32_t kb0, kb;                 // blocks of the reduction: the first one and how many
};

// The tiles of a launch by their number; a CTA (pair) takes every so many of them, in rising order.
template <int CTAS>
struct Tiles {
    const F8Params &p;
    const int32_t *first, *start;    // [groups + 1] first tile / first row
    const int32_t kb0, kb;           // this CTA's part of the reduction
    int32_t g = 0;
    __device__ __forceinline__ Tiles(const F8Params &p_, const int32_t *f, const int32_t *s, int32_t k0, int32_t k) : p(p_), first(f), start(s), kb0(k0), kb(k) {}
    // (without offsets there is one group of all rows, and nothing to look up)
    __device__ __forceinline__ int32_t count() const { return p.offsets ? first[p.groups] : p.tiles_c * p.chunks; }
    __device__ __forceinline__ F8Tile at(int32_t t)
    {
        F8Tile r;
        int32_t i = t, s0 = 0, s1 = (int32_t)p.M;
        if (p.offsets) {
            while (t >= first[g + 1]) ++g;
            i -= first[g];
            s0 = start[g]; s1 = start[g + 1];
        }
        r.g = g;
        const int32_t len = s1 - s0;
        int32_t chunks = p.chunks, csize = p.chunk;
        if (p.offsets) {
            chunks = (len + p.nt - 1) / p.nt;
            csize = ((len + chunks - 1) / chunks + p.step - 1) / p.step * p.step;
        }
        // (p.super chunks go through all channels before the next ones)
        const int32_t sup = chunks > p.super ? i / (p.super * p.tiles_c) : 0;
        const int32_t j = i - sup * p.super * p.tiles_c;
        const int32_t wide = chunks - sup * p.super < p.super ? chunks - sup * p.super : p.super;
        const int32_t c = wide == 1 ? j : j / wide;
        const int32_t ch = sup * p.super + (j - c * wide);
        r.c0 = c * BM * CTAS;
        r.m0 = s0 + ch * csize;
        r.cols = s1 - r.m0 < csize ? s1 - r.m0 : csize;
        r.kb0 = kb0;
        r.kb = kb;
        r.n = (r.cols + 15) / 16 * 16;
        return r;
    }
};

// What the roles of a CTA read their tiles from: warp 3 works them out, a tile a lane, 32 at a time into one of two halves.  (Each role
// for itself, the divisions and look-ups of a grouped tile cost the multiplying warp a fifth of a short tile.)
struct TileQueue {
    const int4 *ring;                // two words of four numbers a tile
    uint32_t full, empty;            // barriers of the halves, 8 bytes apart
    volatile int *abort_flag;
    uint32_t i = 0;
    __device__ __forceinline__ TileQueue(const int4 *r, uint32_t f, uint32_t e, volatile int *a) : ring(r), full(f), empty(e), abort_flag(a) {}
    __device__ __forceinline__ bool read(F8Tile &r)
    {
        const int4 u = ring[(i & 63u) * 2u], v = ring[(i & 63u) * 2u + 1u];
        r.g = u.x; r.c0 = u.y; r.m0 = u.z; r.cols = u.w;
        r.n = v.x; r.kb0 = v.y; r.kb = v.z;
        return r.cols > 0;
    }
    // the next tile, for a thread alone; false: there is none (or the block is aborting)
    __device__ __forceinline__ bool next(F8Tile &r)
    {
        const uint32_t half = i >> 5 & 1u;
        if ((i & 31u) == 0 && !mbar_wait(full + 8u * half, i >> 6 & 1u, abort_flag, 50)) return false;
        const bool more = read(r);
        if ((i & 31u) == 31u) mbar_arrive(empty + 8u * half);
        ++i;
        return more;
    }
    // the same for all lanes of a warp
    __device__ __forceinline__ bool next_warp(F8Tile &r)
    {
        const uint32_t half = i >> 5 & 1u;
        if ((i & 31u) == 0 && !warp_wait(full + 8u * half, i >> 6 & 1u, abort_flag, 50)) return false;
        const bool more = read(r);
        if ((i & 31u) == 31u) {
            __syncwarp();
            if ((threadIdx.x & 31) == 0) mbar_arrive(empty + 8u * half);
        }
        ++i;
        return more;
    }
};

// first[], start[] in shared memory from the offsets in global memory, by all threads of the block.  Offsets that fall, or leave
// 0..M, are held to rise and to stay inside, so that no group reaches rows that are not there.
__device__ void fill_tables(const F8Params &p, int32_t *first, int32_t *start, int32_t *scratch)
{
    constexpr int W = F8_THREADS / 32;
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
        if (g <= G) v = __ldg(p.offsets + g);
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
    // tiles of each group, added up
    int32_t tl[PER], tsum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int g = tid * PER + i;
        const int32_t len = g < G ? start[g + 1] - start[g] : 0;
        tl[i] = tsum;
        if (g < G) tsum += (len + p.nt - 1) / p.nt * p.tiles_c;
    }
    int32_t trun = tsum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int32_t v = __shfl_up_sync(0xffffffffu, trun, d);
        if (lane >= d) trun += v;
    }
    if (lane == 31) scratch[W + warp] = trun;
    __syncthreads();
    trun -= tsum;
    for (int w = 0; w < warp; ++w) trun += scratch[W + w];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int g = tid * PER + i;
        if (g <= G) {
            first[g] = trun + tl[i];
        }
    }
    __syncthreads();
}

// ---- the kernel --------------------------------------------------------------------------------------------------

// SPLIT > 1: so many CTAs of a cluster share one tile, each adds up a part of the reduction, and the sums meet in shared memory.
template <int NT, int MODE, int CTAS, typename TOUT, int SPLIT>
__global__ void __launch_bounds__(F8_THREADS, F8Cfg<NT, MODE, CTAS, TOUT, SPLIT>::RESIDENT)
gemm_f8_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_x32,
               const __grid_constant__ CUtensorMap tmap_out,
               const F8Params p)
{
    using S = F8Cfg<NT, MODE, CTAS, TOUT, SPLIT>;
    constexpr bool CUT = S::CUT;
    static_assert(!CUT || (CTAS == 1 && S::STAGES * S::STAGE_BYTES >= NT * BM * 4), "the partial sums reuse the stages");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;                      // swizzled tiles need 1024-byte alignment
    uint8_t *gen = smem_raw + (base - raw);
    const uint32_t bar0 = base + S::BAR_OFFSET;
    auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(S::STAGES + s); };
    auto sfull_bar = [&](int s) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + s); };
    auto tfull_bar = [&](int a) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + 2 + a); };
    auto tempty_bar = [&](int a) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + 4 + a); };
    auto qfull_bar = [&](int s) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + 6 + s); };
    const uint32_t join_bar = bar0 + 8u * (uint32_t)(2 * S::STAGES + 6 + S::QS);
    const uint32_t tiles_full = join_bar + 8u, tiles_empty = join_bar + 24u;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(gen + S::BAR_OFFSET + 8 * (2 * S::STAGES + 11 + S::QS));
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
        for (int a = 0; a < 2; ++a) { mbar_init(sfull_bar(a), 4 * CTAS); mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 8 * CTAS); }
        for (int s = 0; s < S::QS; ++s) mbar_init(qfull_bar(s), 4);
        if (S::PUSH) mbar_init(join_bar, 1);
        // (read by warps 0, 4..15, and 1 where the products are issued)
        for (int h = 0; h < 2; ++h) { mbar_init(tiles_full + 8u * h, 1); mbar_init(tiles_empty + 8u * h, 13 + (leader ? 1 : 0)); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (S::PUSH) expect_tx(join_bar, (uint32_t)(BM * 4 * NT));     // what the CTAs of the cluster send here
    }
    if (warp == 1) tmem_alloc<CTAS>(smem_u32(tmem_slot), S::TMEM);
    if (warp == 2 && lane < 3 && p.has_maps) {
        const CUtensorMap *m = lane == 0 ? &tmap_w : lane == 1 ? &tmap_x : &tmap_x32;
        asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();                                 // the peer's barriers exist before anything arrives on them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    if (S::PUSH) cluster_arrive();                                     // nothing is sent before every CTA's barrier stands
    // only now may the next kernel be scheduled: one that shares this SM could take the tensor memory this CTA waits for
    griddep_launch_dependents();
    griddep_wait();
    if (p.offsets) fill_tables(p, first, start, reinterpret_cast<int32_t *>(gen + S::STG_OFFSET));

    // a part of the reduction is whole words of scales
    const int32_t part_k = CUT ? (int32_t)cluster_ctarank() : 0;
    const int32_t words = (p.nkb + 3) / 4, kb0 = CUT ? words * part_k / SPLIT * 4 : 0;
    const int32_t kb1 = !CUT || part_k == SPLIT - 1 ? p.nkb : words * (part_k + 1) / SPLIT * 4;
    int4 *ring = reinterpret_cast<int4 *>(gen + S::RING_OFFSET);
    TileQueue queue(ring, tiles_full, tiles_empty, abort_flag);

    if (warp == 3) {
        Tiles<CTAS> tiles(p, first, start, kb0, kb1 - kb0);
        const int32_t num_tiles = tiles.count(), workers = (int32_t)(gridDim.x / (CTAS * SPLIT));
        int64_t t = (int64_t)(blockIdx.x / (CTAS * SPLIT)) + (int64_t)lane * workers;
        for (uint32_t b = 0;; ++b, t += 32 * (int64_t)workers) {
            if (b >= 2 && !warp_wait(tiles_empty + 8u * (b & 1u), (b >> 1) - 1u & 1u, abort_flag, 51)) break;
            F8Tile r{};
            if (t < num_tiles) r = tiles.at((int32_t)t);
            int4 *to = ring + (32u * (b & 1u) + (uint32_t)lane) * 2u;
            to[0] = make_int4(r.g, r.c0, r.m0, r.cols);
            to[1] = make_int4(r.n, r.kb0, r.kb, 0);
            __syncwarp();
            if (lane == 0) mbar_arrive(tiles_full + 8u * (b & 1u));
            if (__any_sync(0xffffffffu, t >= num_tiles)) break;
        }
    }

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0; uint32_t phase = 0;
            bool ok = true, ready = false;
            // (shared::cluster addresses)
            const uint32_t fb0 = CTAS == 2 ? map_to_cta(full_bar(0), 0) : full_bar(0), eb0 = empty_bar(0);
            uint32_t sa = base, fb = fb0, eb = eb0;
            for (F8Tile r; ok && queue.next(r);) {
                const int32_t mine = r.n / CTAS;                       // columns this CTA loads
                const int32_t x0 = r.m0 + (int32_t)rank * mine;
                const int32_t c0 = r.c0 + (int32_t)rank * BM;
                // boxes of 128 rows, the rest in boxes of 32
                const int32_t n32 = (mine + 31) / 32;
                const int32_t big = S::BROWS >= 128 ? n32 / 4 + (n32 % 4 == 3 ? 1 : 0) : 0;
                const int32_t small = n32 <= 4 * big ? 0 : n32 - 4 * big;
                const int32_t boxes = big + small;
                const uint32_t bytes = (uint32_t)(S::A_BYTES + big * 128 * BKB + small * 32 * BKB) * CTAS;
                const CUtensorMap *map0 = big > 0 ? &tmap_x : &tmap_x32;
                int32_t k = r.kb0 * BKB;           // along the reduction
#pragma unroll 1
                for (int32_t kb = 0; kb < r.kb; ++kb, k += BKB) {
                    if (!ready && !mbar_wait(eb, phase ^ 1u, abort_flag, 41)) { ok = false; break; }
                    const bool wrap = stage == S::STAGES - 1;
                    const uint32_t sa_n = wrap ? base : sa + (uint32_t)S::STAGE_BYTES;
                    const uint32_t fb_n = wrap ? fb0 : fb + 8u, eb_n = wrap ? eb0 : eb + 8u;
                    const uint32_t phase_n = wrap ? phase ^ 1u : phase;
                    const uint32_t sb = sa + S::A_BYTES;
                    ready = tma_f8_stage<CTAS>(eb_n, phase_n ^ 1u, fb, bytes, (uint32_t)leader, sa, &tmap_w, MODE == FORWARD ? k : c0, MODE == FORWARD ? c0 : k,
                                               r.g, sb, map0, k, x0) != 0;
                    for (int32_t i = 1; i < boxes; ++i) {
                        const int32_t at = i < big ? i * 128 : big * 128 + (i - big) * 32;
                        tma_load_2d<CTAS>(sb + (uint32_t)(at * BKB), i < big ? &tmap_x : &tmap_x32, k, x0 + at, fb);
                    }
                    stage = wrap ? 0 : stage + 1;
                    sa = sa_n; fb = fb_n; eb = eb_n; phase = phase_n;
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && leader) {
            int stage = 0; uint32_t phase = 0, word = 0, iter = 0;
            bool ok = true, ready = false;
            // a step of 32 along the reduction: 32 bytes of a K-major row, 32 rows of an MN-major tile
            constexpr uint32_t A_STEP = MODE == FORWARD ? 2 : (32 * BKB) >> 4, B_STEP = 2;
            const uint64_t ad = MODE == FORWARD ? make_kmajor_desc<BKB>(base) : make_across_desc(base);
            const uint64_t bd = make_kmajor_desc<BKB>(base + S::A_BYTES);
            const uint32_t a_hi = (uint32_t)(ad >> 32), b_hi = (uint32_t)(bd >> 32), a_lo0 = (uint32_t)ad, fb0 = full_bar(0), eb0 = empty_bar(0);
            const uint32_t b_off = (uint32_t)bd - (uint32_t)ad;
            uint32_t a_lo = a_lo0, fb = fb0, eb = eb0;
            F8Tile r, after;
            bool sready = false, more = queue.next(r);
            for (bool next_more = false; more && ok; more = next_more, r = after, ++iter) {
                const uint32_t as = iter & 1u, aphase = (iter >> 1) & 1u;
                // the accumulator's last tile has been read; where the two share columns, those of the last tile have
                if (p.overlap ? iter > 0 && !mbar_wait(tempty_bar(0), iter - 1u & 1u, abort_flag, 42)
                              : !mbar_wait(tempty_bar(as), aphase ^ 1u, abort_flag, 42)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + (as ? (uint32_t)p.acc1 : 0u);
                const uint32_t idesc = p.idesc | (uint32_t)(r.n >> 3) << 17;
                uint32_t sf = 0;
#pragma unroll 4
                for (int32_t kb = 0; kb < r.kb; ++kb) {
                    if ((kb & 3) == 0) {
                        if (!sready && !mbar_wait(sfull_bar((int)(word & 1u)), word >> 1 & 1u, abort_flag, 43)) { ok = false; break; }
                        sready = false;
                        sf = tmem_base + S::SF_BASE + (word & 1u) * S::SF_COLS;
                        ++word;
                    }
                    if (!ready && !mbar_wait(fb, phase, abort_flag, 44)) { ok = false; break; }
                    tc_fence_after();
                    const bool wrap = stage == S::STAGES - 1;
                    const uint32_t a_lo_n = wrap ? a_lo0 : a_lo + (uint32_t)(S::STAGE_BYTES >> 4);
                    const uint32_t fb_n = wrap ? fb0 : fb + 8u, eb_n = wrap ? eb0 : eb + 8u;
                    const uint32_t phase_n = wrap ? phase ^ 1u : phase;
                    // (bits 4..5 and 29..30: which byte of the scales' words)
                    ready = umma_f8_block<CTAS, A_STEP, B_STEP>(fb_n, phase_n, d_tmem, a_lo, a_hi, a_lo + b_off, b_hi,
                                                                idesc | (uint32_t)(kb & 3) << 29 | (uint32_t)(kb & 3) << 4, (uint32_t)(kb != 0), sf, eb) != 0;
                    stage = wrap ? 0 : stage + 1;
                    a_lo = a_lo_n; fb = fb_n; eb = eb_n; phase = phase_n;
                    // (behind the issue: the next tile's numbers, and whether the next word of scales is there)
                    if (kb == 0) next_more = queue.next(after);
                    if ((kb & 3) == 2) sready = mbar_test(sfull_bar((int)(word & 1u)), word >> 1 & 1u);
                }
                if (r.kb == 0) next_more = queue.next(after);
                if (ok) commit<CTAS>(tfull_bar(as));                   // accumulator complete
            }
        }
    } else if (warp >= 12) {
        // Scales: a word holds four blocks' bytes of a row; word r of a piece of 128 rows goes to lane r % 32 of column r / 32, the same in
        // each quarter of the lanes, one warp a quarter.  Two words have room.  A word's room is free when the products of the word before
        // the last one are done: their last stage's barrier tells.
        const uint32_t tsf = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + S::SF_BASE;
        const uint32_t sfull0 = CTAS == 2 ? map_to_cta(sfull_bar(0), 0) : sfull_bar(0);
        uint32_t word = 0;
        int stage = 0, last1 = 0, last2 = 0;                           // the next block's stage, those of the last blocks of the last two words
        uint32_t phase = 0, phase1 = 0, phase2 = 0;
        int slot = 0; uint32_t qphase = 0;
        bool ok = true;
        // w: 4 words of the tile's rows, then 4 for each 128 columns
        auto put = [&](const uint32_t *w, int blocks) {
            if (word >= 2 && !warp_wait(empty_bar(last2), phase2, abort_flag, 45)) return false;
            tc_fence_after();
            const uint32_t dst = tsf + (word & 1u) * S::SF_COLS;
#pragma unroll
            for (int i = 0; i <= S::SFB; ++i) tmem_st4(dst + 4u * (uint32_t)i, w + 4 * i);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at_leader<CTAS>(sfull0 + 8u * (word & 1u));
            ++word;
            stage += blocks - 1;
            if (stage >= S::STAGES) { stage -= S::STAGES; phase ^= 1u; }
            last2 = last1; phase2 = phase1;
            last1 = stage; phase1 = phase;
            if (++stage == S::STAGES) { stage = 0; phase ^= 1u; }
            return true;
        };
        if (kb1 <= kb0) {
            for (F8Tile r; queue.next_warp(r);) {}                     // (an empty reduction: nothing to scale)
        } else if (F8Tile r; queue.next_warp(r)) {
            // Sixteen blocks' bytes at a time: each warp fetches a quarter of the columns', the next ones while these are used, and all
            // four read the others' from shared memory.  (Each fetching all of them costs the pipe that feeds the tensor core an eighth
            // of its time, and 16-byte boxes by TMA take the loads' turns.)
            // With up to 64 columns each fetches all of them.
            constexpr int R = (NT + 31) / 32;                          // groups of 32 columns
            constexpr bool ALONE = R <= 2;
            constexpr int RW = ALONE ? R : (R + 3) / 4, EVERY = ALONE ? 1 : 4;         // those of a warp
            const int w4 = ALONE ? 0 : warp & 3;
            uint4 mine[RW], a;
            auto fetch = [&](const F8Tile &r, int32_t kb) {
#pragma unroll
                for (int i = 0; i < RW; ++i) {
                    const int32_t row = 32 * (w4 + EVERY * i) + lane;
                    mine[i] = row < r.cols ? ldg128(p.x_scale + (int64_t)(r.m0 + row) * p.ld_xs + kb) : make_uint4(0, 0, 0, 0);
                }
                const int32_t ct = (r.c0 + (int32_t)rank * BM) / BM;
                const bool has_ct = ct * BM < p.N;                     // (a pair's second half may lie beyond the channels)
                const uint8_t *ws = p.w_scale + (int64_t)r.g * p.stride_ws;
                a = make_uint4(0, 0, 0, 0);
                if (MODE == FORWARD) {
                    if (has_ct) a = ldg128(ws + (int64_t)ct * p.ld_ws + kb);
                } else {
                    if (lane < 16 && has_ct && kb + lane < kb1) a.x = ws[(int64_t)(kb + lane) * p.ld_ws + ct];
                }
            };
            int32_t kb = kb0 & ~15;                                    // (16 bytes lie on 16 bytes)
            fetch(r, kb);
            for (bool more = true; more && ok;) {
                uint4 *qs = reinterpret_cast<uint4 *>(gen + S::Q_OFFSET + slot * S::Q_BYTES) + lane;
                if (!ALONE) {
#pragma unroll
                    for (int i = 0; i < RW; ++i)
                        if (32 * (w4 + 4 * i) + lane < NT) qs[32 * (w4 + 4 * i)] = mine[i];
                }
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
                uint4 x[R];
                if constexpr (ALONE) {
#pragma unroll
                    for (int i = 0; i < R; ++i) x[i] = mine[i];
                } else {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(qfull_bar(slot));
                    if (!warp_wait(qfull_bar(slot), qphase, abort_flag, 48)) break;
#pragma unroll
                    for (int i = 0; i < R; ++i) x[i] = 32 * i + lane < NT ? qs[32 * i] : make_uint4(0, 0, 0, 0);
                    // (two slots: before a warp writes this one again, all have passed the other's barrier, and so have read this one)
                    if (++slot == 2) { slot = 0; qphase ^= 1u; }
                }
                const int32_t skip = kb < kb0 ? kb0 - kb : 0, blocks = kb1 - kb;
                kb += 16;
                if (kb >= kb1) {
                    kb = kb0 & ~15;
                    more = queue.next_warp(r);
                }
                if (more) fetch(r, kb);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int left = blocks - 4 * j;
                    if (left <= 0 || !ok) break;
                    if (4 * j < skip) continue;
                    uint32_t w[S::SF_COLS];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = aw[j];
#pragma unroll
                    for (int i = 0; i < 4 * S::SFB; ++i) w[4 + i] = i < R ? (j == 0 ? x[i < R ? i : 0].x : j == 1 ? x[i < R ? i : 0].y : j == 2 ? x[i < R ? i : 0].z : x[i < R ? i : 0].w) : 0u;
                    ok = put(w, left < 4 ? left : 4);
                }
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3, part = (warp - 4) >> 2;                // tensor-memory lane quarter this warp may read; even or odd blocks of columns
        uint8_t *stg = gen + S::STG_OFFSET + (warp - 4) * 32 * 32 * (int)sizeof(TOUT);
        constexpr int EPV = 16 / (int)sizeof(TOUT);                    // elements of a 16-byte piece
        constexpr int PIECES = 32 / EPV;                               // pieces of a staged row
        constexpr int PITCH = 32 * (int)sizeof(TOUT);
        // 16-byte pieces of a staged row change places with the row, so that rows written by 32 lanes at once meet in no bank
        auto swz = [](int row, int piece) { return sizeof(TOUT) == 4 ? piece ^ (row & 7) : piece ^ ((row >> 1) & 3); };
        if (S::PUSH) cluster_wait();
        uint32_t iter = 0;
        for (F8Tile r; queue.next_warp(r); ++iter) {
            const uint32_t as = iter & 1u, aphase = (iter >> 1) & 1u;
            const int32_t ch = r.c0 + (int32_t)rank * BM + q * 32;     // the channel of the warp's first row of tensor memory
            const float bias = p.bias && ch + lane < p.N ? __ldg(p.bias + (int64_t)r.g * p.N + ch + lane) : 0.0f;
            // the tensor-memory loads below are warp-collective: leave the loop only as a whole warp
            if (!warp_wait(tfull_bar(as), aphase, abort_flag, 46)) break;
            tc_fence_after();
            const uint32_t tacc = tmem_base + ((uint32_t)(q * 32) << 16) + (as ? (uint32_t)p.acc1 : 0u);
            const int32_t nblk = CUT || ch < p.N ? (r.cols + 31) / 32 : 0;       // (warp-uniform)
            // Blocks of columns in rising order; the first accumulator's, if its last block is shared, in falling order.
            const bool falling = p.overlap && as == 0;
            bool shared = p.overlap != 0;                              // not yet handed back
            auto staged_block_read = [&]() {                           // the block before has left shared memory
                if (lane == 0) bulk_wait_read<0>();
                __syncwarp();
            };
            auto hand_back = [&](uint32_t bar) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at_leader<CTAS>(CTAS == 2 ? map_to_cta(bar, 0) : bar);
            };
            const int32_t last = (nblk - 1) | 1;
            for (int32_t i = part; i <= last; i += 2) {
                const int32_t b = falling ? last - i : i;
                if (b >= nblk) continue;
                uint32_t v[32];
                if constexpr (S::PUSH) {
                    // CTA d of the cluster joins columns d * OWN .. of the tile; a few columns of a channel are sent at a time
                    constexpr int OWN = NT / SPLIT, W = OWN < 4 ? OWN : 4;
                    tmem_ld32(tacc, v);
                    const uint32_t to = base + (uint32_t)(S::JOIN_OFFSET + (part_k * BM + q * 32 + lane) * OWN * 4);
#pragma unroll
                    for (int d = 0; d < SPLIT; ++d) {
                        const uint32_t at = map_to_cta(to, (uint32_t)d), bar = map_to_cta(join_bar, (uint32_t)d);
#pragma unroll
                        for (int j = 0; j < OWN; j += W) send<W>(at + 4u * (uint32_t)j, v + d * OWN + j, bar);
                    }
                    continue;
                } else if constexpr (CUT) {
                    // this CTA's sums over the operand stages, which nothing reads any more: channels next to each other
                    tmem_ld32(tacc + (uint32_t)(b * 32), v);
                    float *sums = reinterpret_cast<float *>(gen) + b * 32 * BM + q * 32 + lane;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (b * 32 + j < NT) sums[j * BM] = __uint_as_float(v[j]);
                    continue;
                }
                if constexpr (sizeof(TOUT) == 2) {
                    // Channels along lanes become channels along a row: blocks of 8 x 8 in fragments (lane 4 c + t: channel c, columns 2 t
                    // and 2 t + 1), stored transposed.
                    if (r.kb > 0) tmem_ld_frag(tacc + (uint32_t)(b * 32), v);
                    if (shared) { hand_back(tempty_bar(0)); shared = false; }
                    float bi[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) bi[i] = __shfl_sync(0xffffffffu, bias, 8 * i + (lane >> 2));
                    staged_block_read();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {                      // columns 8 c .. 8 c + 7
                        uint32_t o[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {                  // channels 8 i .. 8 i + 7
                            const int at = (i >> 1) * 16 + 4 * c + 2 * (i & 1);
                            o[i] = r.kb > 0 ? pack2(__uint_as_float(v[at]) + bi[i], __uint_as_float(v[at + 1]) + bi[i], TOUT()) : pack2(bi[i], bi[i], TOUT());
                        }
                        const int row = 8 * c + (lane & 7);
                        stmatrix_trans(smem_u32(stg + row * PITCH + swz(row, lane >> 3) * 16), o);
                    }
                } else {
                    if (r.kb > 0) tmem_ld32(tacc + (uint32_t)(b * 32), v);
                    if (shared) { hand_back(tempty_bar(0)); shared = false; }
                    float f[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] = r.kb > 0 ? __uint_as_float(v[j]) + bias : bias;
                    staged_block_read();
                    // lanes are channels, next to each other in the output's rows
#pragma unroll
                    for (int j = 0; j < 32; ++j) *reinterpret_cast<float *>(stg + j * PITCH + swz(j, lane / 4) * 16 + (lane % 4) * 4) = f[j];
                }
                // the staged block: `rows` rows of `cols` elements at dst
                const int32_t rows_left = r.cols - b * 32, cols_left = p.N - ch;
                const int rows = rows_left < 32 ? rows_left : 32, cols = cols_left < 32 ? cols_left : 32;
                TOUT *dst = static_cast<TOUT *>(p.out) + (int64_t)(r.m0 + b * 32) * p.ldo + ch;
                // A bulk store writes the whole block, but for what lies behind the matrix.
                if (p.tma_out && (rows == 32 || r.m0 + b * 32 + rows == p.M)) {
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_3d(&tmap_out, ch, r.m0 + b * 32, 0, smem_u32(stg));
                        bulk_commit();
                    }
                    continue;
                }
                __syncwarp();
                if (p.vec_out && cols == 32) {
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) {
                        const int row = i * (32 / PIECES) + lane / PIECES, c = lane % PIECES;
                        const uint4 o = *reinterpret_cast<const uint4 *>(stg + row * PITCH + swz(row, c) * 16);
                        if (row < rows) *reinterpret_cast<uint4 *>(dst + (int64_t)row * p.ldo + c * EPV) = o;
                    }
                } else {
                    // rows of any alignment: lanes along the row, element by element
                    TOUT *d = dst + lane;
#pragma unroll
                    for (int r0 = 0; r0 < 32; r0 += 8) {
                        TOUT o[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            o[i] = *reinterpret_cast<const TOUT *>(stg + (r0 + i) * PITCH + swz(r0 + i, lane / EPV) * 16 + (lane % EPV) * (int)sizeof(TOUT));
#pragma unroll
                        for (int i = 0; i < 8; ++i, d += p.ldo)
                            if (r0 + i < rows && lane < cols) *d = o[i];
                    }
                }
            }
            // all reads of this accumulator are done (where columns are shared: this warp has none to read, or has read them)
            if (shared || !p.overlap) hand_back(p.overlap ? tempty_bar(0) : tempty_bar(as));
        }
        if (lane == 0) bulk_wait_all();                                // stores must have read shared memory before it goes away
        __syncwarp();
    }

    __syncwarp();
    if (*abort_flag) let_flights_land();
    tc_fence_before();
    if constexpr (S::PUSH) {
        if (warp < 4 || warp >= 12) cluster_wait();                    // (the storing warps have)
        if (warp >= 4 && warp < 8) {
            // sums of this CTA's columns, in the order of the parts of the reduction
            constexpr int OWN = NT / SPLIT;
            F8Tile r;
            queue.i = 0;                                               // (the cluster's only tile)
            queue.read(r);
            const int ch0 = (warp & 3) * 32 + lane, ch = r.c0 + ch0;
            const float bias = p.bias && ch < p.N ? __ldg(p.bias + ch) : 0.0f;
            if (warp_wait(join_bar, 0, abort_flag, 49)) {
                float sum[OWN];
#pragma unroll
                for (int i = 0; i < SPLIT; ++i) {
                    const float *part = reinterpret_cast<const float *>(gen + S::JOIN_OFFSET) + (i * BM + ch0) * OWN;
#pragma unroll
                    for (int c = 0; c < OWN; ++c) sum[c] = i == 0 ? part[c] : sum[c] + part[c];
                }
                TOUT *dst = static_cast<TOUT *>(p.out) + (int64_t)(r.m0 + part_k * OWN) * p.ldo + ch;
#pragma unroll
                for (int c = 0; c < OWN; ++c)
                    if (ch < p.N && part_k * OWN + c < r.cols) from_float(sum[c] + bias, dst[c * p.ldo]);
            }
        }
        // a CTA whose wait ran out must not end while others may still send to it
        __syncthreads();
        if (*abort_flag) stay_for_cluster();
    } else if constexpr (CUT) {
        // every CTA joins a part of the columns, in the order of the parts of the reduction, and stays until the others have read its sums
        cluster_sync_all();
        F8Tile r;
        queue.i = 0;                                                   // (the cluster's only tile)
        queue.read(r);
        const int32_t mine0 = r.cols * part_k / SPLIT, mine1 = r.cols * (part_k + 1) / SPLIT;
        const int32_t ch = r.c0 + lane * 4;
        float bias[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[i] = p.bias && ch + i < p.N ? __ldg(p.bias + ch + i) : 0.0f;
        for (int32_t c = mine0 + warp; c < mine1; c += F8_THREADS / 32) {
            const uint32_t at = base + (uint32_t)(c * BM + lane * 4) * 4u;
            float4 v[SPLIT];
#pragma unroll
            for (int i = 0; i < SPLIT; ++i) v[i] = ld_peer_f32x4(map_to_cta(at, (uint32_t)i));
            float4 sum = v[0];
#pragma unroll
            for (int i = 1; i < SPLIT; ++i) { sum.x += v[i].x; sum.y += v[i].y; sum.z += v[i].z; sum.w += v[i].w; }
            TOUT *dst = static_cast<TOUT *>(p.out) + (int64_t)(r.m0 + c) * p.ldo + ch;
            const float f[4] = {sum.x + bias[0], sum.y + bias[1], sum.z + bias[2], sum.w + bias[3]};
            if (p.vec_out && ch + 4 <= p.N) {
                if constexpr (sizeof(TOUT) == 4) *reinterpret_cast<float4 *>(dst) = make_float4(f[0], f[1], f[2], f[3]);
                else *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2(f[0], f[1], TOUT()), pack2(f[2], f[3], TOUT()));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (ch + i < p.N) from_float(f[i], dst[i]);
            }
        }
        cluster_sync_all();
    }
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();     // the peer no longer touches this CTA's barriers, shared or tensor memory
    tc_fence_after();
    if (warp == 1) tmem_dealloc<CTAS>(tmem_base, S::TMEM);
}

// ---- host --------------------------------------------------------------------------------------------------------

int make_map_f8(const char *what, CUtensorMap *map, const void *ptr, int dims_n, int64_t cols, int64_t rows, int64_t count, int64_t ld, int64_t stride,
                int box_cols, int box_rows, CUtensorMapSwizzle swizzle, CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_UINT8)
{
    EncodeTiledFn fn = encode_fn();
    QNN_REQUIRE(fn != nullptr, QNN_ERR_CUDA, "%s: cuTensorMapEncodeTiled is not available from this driver", what);
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)count};
    cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)stride};
    cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    CUresult r = fn(map, type, (cuuint32_t)dims_n, const_cast<void *>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    QNN_REQUIRE(r == CUDA_SUCCESS, QNN_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed with code %d", what, (int)r);
    return QNN_OK;
}

template <int NT, int MODE, int CTAS, typename TOUT, int SPLIT = 1>
int launch_f8(const F8Call &c, F8Params p, const F8Choice &how, cudaStream_t st)
{
    using S = F8Cfg<NT, MODE, CTAS, TOUT, SPLIT>;
    auto kern = gemm_f8_kernel<NT, MODE, CTAS, TOUT, SPLIT>;
    constexpr int STEP = chunk_step(NT);
    static_assert(NT % STEP == 0, "a chunk is never wider than a tile");
    p.step = STEP;
    p.nt = how.nt;
    p.tiles_c = (int32_t)ceil_div(p.N, BM * CTAS);
    p.overlap = 2 * p.nt > S::SF_BASE;
    p.acc1 = p.overlap ? NT - 32 : S::SF_BASE / 32 * 16;
    p.chunk = p.nt;
    p.chunks = (int32_t)ceil_div(p.M, p.chunk);
    p.super = 16;
    const int64_t tiles = (p.chunks + (p.offsets ? p.groups : 0)) * (int64_t)p.tiles_c;
    QNN_REQUIRE(tiles < (int64_t)1 << 28, QNN_ERR_UNSUPPORTED, "%s: too many output tiles", c.what);
    static std::atomic<bool> done[64];
    if (int rc = opt_in(kern, S::TOTAL, done)) return rc;
    CUtensorMap mw{}, mx{}, mx32{}, mo{};
    // (an empty reduction loads nothing: any map will do)
    const bool empty = c.w_rows == 0 || c.w_cols == 0 || c.x_rows == 0 || c.x_cols == 0;
    p.has_maps = !empty;
    if (!empty) {
        const CUtensorMapSwizzle wide = CU_TENSOR_MAP_SWIZZLE_128B;
        if (int rc = make_map_f8(c.what, &mw, c.w, 3, c.w_cols, c.w_rows, c.w_count, c.ld_w, c.stride_w, BKB, BM, wide)) return rc;
        if (int rc = make_map_f8(c.what, &mx, c.x, 2, c.x_cols, c.x_rows, 1, c.ld_x, 0, BKB, 128, wide)) return rc;
        if (int rc = make_map_f8(c.what, &mx32, c.x, 2, c.x_cols, c.x_rows, 1, c.ld_x, 0, BKB, 32, wide)) return rc;
    }
    {
        // (a bulk store clips a row in 16-byte units)
        const int64_t es = (int64_t)sizeof(TOUT), cols = p.N, rows = p.M;
        const int64_t ld = p.ldo * es, stride = ld;
        p.tma_out = !S::CUT && p.vec_out && cols * es % 16 == 0 && ld < (int64_t)1 << 40 && stride < (int64_t)1 << 40;
        if (p.tma_out)
            if (int rc = make_map_f8(c.what, &mo, p.out, 3, cols, rows, 1, ld, stride, 32, 32, es == 4 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                     es == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16)) return rc;
    }
    // operand types, which dimension is contiguous, scales as powers of two, rows of the tile
    p.idesc = (uint32_t)c.w_type << 7 | (uint32_t)c.x_type << 10 | (MODE != FORWARD ? 1u : 0u) << 15 | 1u << 23 |
              (uint32_t)((BM * CTAS) >> 7) << 27;
    const int64_t resident = CTAS == 2 ? pairs_resident_f8() : sm_count();
    const int64_t ctas = S::CUT ? tiles * SPLIT : CTAS * (tiles < resident ? tiles : resident);
    constexpr unsigned cluster = CTAS * SPLIT;
    profile_before(st);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas); cfg.blockDim = dim3(F8_THREADS); cfg.dynamicSmemBytes = S::TOTAL; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    unsigned na = 0;
    if (cluster > 1) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = cluster; attr[na].val.clusterDim.y = 1; attr[na].val.clusterDim.z = 1;
        ++na;
    }
    if (pdl_enabled()) {
        attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[na].val.programmaticStreamSerializationAllowed = 1;
        ++na;
    }
    cfg.attrs = attr; cfg.numAttrs = na;
    QNN_CUDA(cudaLaunchKernelEx(&cfg, kern, mw, mx, mx32, mo, p));
    profile_after(st);
    return check_launch(c.what);
}

template <int NT, int MODE, typename TOUT>
int launch_split(const F8Call &c, const F8Params &p, const F8Choice &k, cudaStream_t st)
{
    switch (k.split) {
        case 2: return launch_f8<NT, MODE, 1, TOUT, 2>(c, p, k, st);
        case 4: return launch_f8<NT, MODE, 1, TOUT, 4>(c, p, k, st);
        default: return launch_f8<NT, MODE, 1, TOUT, 8>(c, p, k, st);
    }
}

template <int MODE, typename TOUT>
int run_f8_typed(const F8Call &c, const F8Params &p, cudaStream_t st)
{
    const F8Choice k = choose_f8(p.M, p.groups, p.N, p.nkb, p.offsets == nullptr);
    if (k.split > 1) return k.width == 16   ? launch_split<16, MODE, TOUT>(c, p, k, st)
                            : k.width == 64 ? launch_split<64, MODE, TOUT>(c, p, k, st)
                                            : launch_split<128, MODE, TOUT>(c, p, k, st);
    switch (k.width) {
        case 32: return launch_f8<32, MODE, 1, TOUT>(c, p, k, st);
        case 64: return launch_f8<64, MODE, 1, TOUT>(c, p, k, st);
        case 128: return launch_f8<128, MODE, 1, TOUT>(c, p, k, st);
        default: return launch_f8<256, MODE, 2, TOUT>(c, p, k, st);
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

}  // namespace
}  // namespace qnn
