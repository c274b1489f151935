// Real values -> 8-bit floating-point codes (e4m3 or e5m2) with a power-of-two scale for each block of 128 elements of a row, 128 x 128
// of a matrix, or 128 rows of a column: the operands of the products in qnn_gemm_f8.cu.
//
// The scale is the least power of two at which the block's largest magnitude fits the codes: read off the exponent and the mantissa
// of that magnitude, so dividing by it is exact and a code is one rounding of the value (to nearest, ties to even).
//
// All of it is bound by memory: every element is read once into registers, the blocks' maxima are joined across lanes (rows: 16 lanes
// hold a block) or through shared memory (tiles, columns), and codes, scales and values are written from the registers.
#include "qnn_types.cuh"

namespace qnn {
namespace {

constexpr uint32_t MANT_MOST = 0x600000u;        // 1.75: mantissa of the largest code of both types
struct F8Source {
    const void *x; int64_t ldx;
    int64_t rows; int32_t K;
    const int64_t *index; int64_t src_rows;
    uint8_t *codes; int64_t ldq;
    uint8_t *scale; int64_t ld_scale;
    void *values; int values_type; int64_t ld_values;
    int e5m2;
    int vec_values;                              // the values' rows may be written in 16-byte pieces
    const int64_t *offsets; int32_t groups;      // columns
    int32_t log_seg, segs;                       // rows: blocks of a warp's part of a row (log2), parts a row
};

// scale byte of a block from the bits of its largest magnitude; an infinity or a NaN gives 255
__device__ __forceinline__ uint32_t scale_byte(uint32_t top, int e5m2)
{
    const int e = (int)(top >> 23), low = e5m2 ? 15 : 8;
    const int s = e - low + ((top & 0x7fffffu) > MANT_MOST ? 1 : 0);
    return e == 255 ? 255u : s < 0 ? 0u : (uint32_t)s;
}
// 1 / scale; 0 for a scale that is NaN, whose codes are 0
__device__ __forceinline__ float scale_inverse(uint32_t s) { return s == 255u ? 0.0f : __uint_as_float((254u - s) << 23); }
__device__ __forceinline__ float scale_value(uint32_t s) { return s == 255u ? __uint_as_float(0x7fffffffu) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23); }

__device__ __forceinline__ uint32_t codes2(float lo, float hi, int e5m2)
{
    uint16_t r;
    if (e5m2) asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 decode2(uint32_t c, int e5m2)
{
    uint32_t h;
    if (e5m2) asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
    else asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
// Eight values of a block with scale byte s: their codes, two a register.  (0 times an infinity is a NaN: such blocks' codes are set.)
__device__ __forceinline__ uint2 encode8(const float (&f)[8], uint32_t s, int e5m2)
{
    const float inv = scale_inverse(s);
    uint2 q;
    q.x = codes2(f[0] * inv, f[1] * inv, e5m2) | codes2(f[2] * inv, f[3] * inv, e5m2) << 16;
    q.y = codes2(f[4] * inv, f[5] * inv, e5m2) | codes2(f[6] * inv, f[7] * inv, e5m2) << 16;
    return s == 255u ? make_uint2(0u, 0u) : q;
}
__device__ __forceinline__ void decode8(uint2 q, float scale, int e5m2, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 d = decode2((i < 2 ? q.x : q.y) >> (16 * (i & 1)) & 0xffffu, e5m2);
        f[2 * i] = d.x * scale; f[2 * i + 1] = d.y * scale;
    }
}
template <typename V>
__device__ __forceinline__ void put_values(V *v, const float (&f)[8], int n, int vec)
{
    if (vec && n >= 8) store_floats<V, 8>(v, f);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) from_float(f[i], v[i]);
}
// what the codes stand for: n elements of a row from (row, k) on
__device__ __forceinline__ void write_values(const F8Source &p, int64_t row, int32_t k, const float (&f)[8], int n)
{
    const int64_t at = row * p.ld_values + k;
    switch (p.values_type) {
        case QNN_TYPE_F32: put_values(static_cast<float *>(p.values) + at, f, n, p.vec_values); break;
        case QNN_TYPE_BF16: put_values(static_cast<__nv_bfloat16 *>(p.values) + at, f, n, p.vec_values); break;
        default: put_values(static_cast<__half *>(p.values) + at, f, n, p.vec_values); break;
    }
}
// eight elements of a row from k on, 0 where it has ended (or is not there)
template <typename T, bool VEC>
__device__ __forceinline__ void read8(const T *row, int32_t k, int32_t K, float (&f)[8])
{
    if (row != nullptr && VEC && k + 8 <= K) {
        Piece<T, 8> v;
        load_piece<T, 8>(row + k, v);
        piece_to_floats<T, 8>(v, f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = row != nullptr && k + i < K ? to_float(row[k + i]) : 0.0f;
    }
}
__device__ __forceinline__ uint32_t magnitude(float f) { return __float_as_uint(f) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t top8(const float (&f)[8])
{
    uint32_t t = magnitude(f[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) t = max(t, magnitude(f[i]));
    return t;
}

// ---- blocks of a row ---------------------------------------------------------------------------------------------

constexpr int ROW_UNITS = 4;                     // blocks a half warp has in flight

// A warp takes eight blocks: 2^log_seg next to each other of each of 8 / 2^log_seg rows; 16 lanes hold a block, eight elements each.
template <typename T, bool VEC>
__global__ void __launch_bounds__(128)
quant_rows_f8_kernel(const F8Source p)
{
    const int lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int64_t rg = w / p.segs;
    const int32_t seg = (int32_t)(w - rg * p.segs);
    const int32_t K16 = (p.K + 15) & ~15;
    griddep_wait();
    float f[ROW_UNITS][8];
#pragma unroll
    for (int u = 0; u < ROW_UNITS; ++u) {
        const int j = 2 * u + half;
        const int64_t row = (rg << (3 - p.log_seg)) + (j >> p.log_seg);
        const int32_t k = (((seg << p.log_seg) + (j & ((1 << p.log_seg) - 1))) << 7) + 8 * l16;
        const T *src = nullptr;
        if (row < p.rows && k < p.K) {
            int64_t from = row;
            if (p.index) from = __ldg(p.index + row);
            if (from >= 0 && (!p.index || from < p.src_rows)) src = static_cast<const T *>(p.x) + from * p.ldx;
        }
        read8<T, VEC>(src, k, p.K, f[u]);
    }
    griddep_launch_dependents();
#pragma unroll
    for (int u = 0; u < ROW_UNITS; ++u) {
        const int j = 2 * u + half;
        const int64_t row = (rg << (3 - p.log_seg)) + (j >> p.log_seg);
        const int32_t blk = (seg << p.log_seg) + (j & ((1 << p.log_seg) - 1)), k = (blk << 7) + 8 * l16;
        uint32_t top = top8(f[u]);
#pragma unroll
        for (int d = 8; d > 0; d /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
        if (row >= p.rows || k >= K16) continue;
        const uint32_t s = scale_byte(top, p.e5m2);
        const uint2 q = encode8(f[u], s, p.e5m2);
        *reinterpret_cast<uint2 *>(p.codes + row * p.ldq + k) = q;
        if (l16 == 0) p.scale[row * p.ld_scale + blk] = (uint8_t)s;
        if (p.values && k < p.K) {
            float v[8];
            decode8(q, scale_value(s), p.e5m2, v);
            write_values(p, row, k, v, p.K - k);
        }
    }
}

// ---- tiles of 128 x 128, and blocks of 128 rows of a column ------------------------------------------------------

// The rows of block b of groups whose rows are filled up to whole blocks: first row, rows left from it on, or -1 where there is no such
// block.  By one warp.  Offsets that fall, or leave 0..M, are held to rise and to stay inside.
__device__ __forceinline__ void find_block(const int64_t *offsets, int32_t groups, int64_t M, int32_t b, int lane, int64_t &row0, int64_t &rows)
{
    row0 = -1; rows = 0;
    int64_t top = 0;                             // running maximum of the offsets
    int32_t before = 0;                          // blocks of the groups before
    for (int32_t g0 = 0; g0 < groups; g0 += 32) {
        const int32_t g = g0 + lane;
        int64_t e = 0;                           // the group's end
        if (g < groups) e = offsets ? __ldg(offsets + g + 1) : M;
        int64_t s0 = 0;
        if (g0 == 0 && offsets) s0 = __ldg(offsets);
        s0 = s0 < 0 ? 0 : s0 > M ? M : s0;
        if (g0 == 0) top = s0;
        e = e < top ? top : e > M ? M : e;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int64_t v = __shfl_up_sync(0xffffffffu, e, d);
            if (lane >= d && v > e) e = v;
        }
        int64_t s = __shfl_up_sync(0xffffffffu, e, 1);
        if (lane == 0) s = top;
        const int32_t mine = g < groups ? (int32_t)((e - s + 127) / 128) : 0;
        int32_t run = mine;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int32_t v = __shfl_up_sync(0xffffffffu, run, d);
            if (lane >= d) run += v;
        }
        const int32_t first = before + run - mine;
        const unsigned hit = __ballot_sync(0xffffffffu, b >= first && b < first + mine);
        if (hit) {
            const int src = __ffs(hit) - 1;
            const int64_t start = s + (int64_t)(b - first) * 128;
            row0 = __shfl_sync(0xffffffffu, start, src);
            rows = __shfl_sync(0xffffffffu, e, src) - row0;
            return;
        }
        before += __shfl_sync(0xffffffffu, run, 31);
        top = __shfl_sync(0xffffffffu, e, 31);
    }
}

constexpr int TILE_THREADS = 256;

// 128 rows x 128 columns a block: 16 lanes hold a row's 128 columns, eight each, and a thread every sixteenth row.
template <typename T, bool VEC, bool COLUMNS>
__global__ void __launch_bounds__(TILE_THREADS)
quant_tiles_f8_kernel(const F8Source p)
{
    __shared__ uint32_t tops[8][128];
    __shared__ __align__(8) uint8_t bytes[128];
    __shared__ int64_t where[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, l16 = tid & 15, r16 = tid >> 4;
    const int32_t tile = blockIdx.x, blk = blockIdx.y;
    const int32_t k = tile * 128 + 8 * l16;
    const int32_t K16 = (p.K + 15) & ~15;
    griddep_wait();
    int64_t row0 = (int64_t)blk * 128, left = p.rows - row0;
    if (COLUMNS) {
        if (warp == 0) {
            find_block(p.offsets, p.groups, p.rows, blk, lane, row0, left);
            if (lane == 0) { where[0] = row0; where[1] = left; }
        }
        __syncthreads();
        row0 = where[0]; left = where[1];
        if (row0 < 0) return;
    }
    const int rows = left < 128 ? (int)left : 128;
    const T *src = static_cast<const T *>(p.x) + row0 * p.ldx;
    float f[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i * 16 + r16;
        read8<T, VEC>(r < rows ? src + (int64_t)r * p.ldx : nullptr, k, p.K, f[i]);
    }
    griddep_launch_dependents();
    uint32_t s[8];
    if (COLUMNS) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            uint32_t t = magnitude(f[0][c]);
#pragma unroll
            for (int i = 1; i < 8; ++i) t = max(t, magnitude(f[i][c]));
            t = max(t, __shfl_xor_sync(0xffffffffu, t, 16));
            s[c] = t;
        }
        if (lane < 16) {
            *reinterpret_cast<uint4 *>(&tops[warp][8 * l16]) = make_uint4(s[0], s[1], s[2], s[3]);
            *reinterpret_cast<uint4 *>(&tops[warp][8 * l16 + 4]) = make_uint4(s[4], s[5], s[6], s[7]);
        }
        __syncthreads();
        if (tid < 128) {
            uint32_t t = tops[0][tid];
#pragma unroll
            for (int w = 1; w < 8; ++w) t = max(t, tops[w][tid]);
            const uint32_t b = scale_byte(t, p.e5m2);
            bytes[tid] = (uint8_t)b;
            if (tile * 128 + tid < p.K) p.scale[(int64_t)blk * p.ld_scale + tile * 128 + tid] = (uint8_t)b;
        }
        __syncthreads();
        const uint2 b8 = *reinterpret_cast<const uint2 *>(&bytes[8 * l16]);
#pragma unroll
        for (int c = 0; c < 8; ++c) s[c] = (c < 4 ? b8.x : b8.y) >> (8 * (c & 3)) & 0xffu;
    } else {
        uint32_t t = top8(f[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) t = max(t, top8(f[i]));
        t = __reduce_max_sync(0xffffffffu, t);
        if (lane == 0) tops[0][warp] = t;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) t = max(t, tops[0][w]);
        const uint32_t b = scale_byte(t, p.e5m2);
        if (tid == 0) p.scale[(int64_t)blk * p.ld_scale + tile] = (uint8_t)b;
#pragma unroll
        for (int c = 0; c < 8; ++c) s[c] = b;
    }
    if (k >= K16) return;
    float inv[8], val[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) { inv[c] = scale_inverse(s[c]); val[c] = scale_value(s[c]); }
    // (columns: the rows that fill a group up to whole blocks are written too, as zeros)
    const int64_t out0 = (int64_t)blk * 128;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i * 16 + r16;
        if (!COLUMNS && r >= rows) continue;
        float g[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) g[c] = s[c] == 255u ? 0.0f : f[i][c] * inv[c];
        uint2 q;
        q.x = codes2(g[0], g[1], p.e5m2) | codes2(g[2], g[3], p.e5m2) << 16;
        q.y = codes2(g[4], g[5], p.e5m2) | codes2(g[6], g[7], p.e5m2) << 16;
        *reinterpret_cast<uint2 *>(p.codes + (out0 + r) * p.ldq + k) = q;
        if (p.values && k < p.K) {
            float v[8];
            decode8(q, 1.0f, p.e5m2, v);
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] *= val[c];
            write_values(p, out0 + r, k, v, p.K - k);
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------------------

enum { BY_ROWS, BY_TILES, BY_COLUMNS };

template <int HOW, typename T>
int launch_quant(F8Source p, const char *what, cudaStream_t st)
{
    const bool vec = aligned(p.x, 16) && (p.ldx * (int64_t)sizeof(T)) % 16 == 0;
    const int64_t nblk = ceil_div(p.K, 128);
    if (HOW == BY_ROWS) {
        p.log_seg = nblk >= 8 ? 3 : nblk > 2 ? 2 : nblk > 1 ? 1 : 0;
        p.segs = (int32_t)ceil_div(nblk, 1 << p.log_seg);
        const int64_t warps = ceil_div(p.rows, 8 >> p.log_seg) * p.segs, blocks = ceil_div(warps, 4);
        QNN_REQUIRE(blocks < (int64_t)1 << 31, QNN_ERR_UNSUPPORTED, "%s: too many blocks", what);
        const dim3 grid((unsigned)blocks);
        if (vec) QNN_CUDA(launch_pdl(quant_rows_f8_kernel<T, true>, grid, dim3(128), 0, st, p));
        else QNN_CUDA(launch_pdl(quant_rows_f8_kernel<T, false>, grid, dim3(128), 0, st, p));
    } else {
        const int64_t blocks = HOW == BY_COLUMNS ? p.rows / 128 + p.groups : ceil_div(p.rows, 128);
        QNN_REQUIRE(blocks < 65536, QNN_ERR_UNSUPPORTED, "%s: 65536 blocks of 128 rows and more", what);
        const dim3 grid((unsigned)nblk, (unsigned)blocks);
        if (vec) QNN_CUDA(launch_pdl(quant_tiles_f8_kernel<T, true, HOW == BY_COLUMNS>, grid, dim3(TILE_THREADS), 0, st, p));
        else QNN_CUDA(launch_pdl(quant_tiles_f8_kernel<T, false, HOW == BY_COLUMNS>, grid, dim3(TILE_THREADS), 0, st, p));
    }
    return check_launch(what);
}

template <int HOW>
int quant_f8(F8Source p, int type, int64_t K, int code_type, const char *what, void *stream)
{
    QNN_REQUIRE(type_ok(type), QNN_ERR_INVALID_ARG, "%s: unknown element type %d", what, type);
    QNN_REQUIRE(code_type == QNN_F8_E4M3 || code_type == QNN_F8_E5M2, QNN_ERR_INVALID_ARG, "%s: unknown type of codes %d", what, code_type);
    QNN_REQUIRE(p.rows >= 0 && K >= 0 && p.src_rows >= 0 && p.groups >= 0, QNN_ERR_INVALID_ARG, "%s: negative size", what);
    if (p.rows == 0 || K == 0) return QNN_OK;
    QNN_REQUIRE(p.rows <= (int64_t)1 << 30 && K <= (int64_t)1 << 30 && p.src_rows <= (int64_t)1 << 30, QNN_ERR_UNSUPPORTED, "%s: a size above 2^30", what);
    QNN_REQUIRE(p.x && p.codes && p.scale, QNN_ERR_INVALID_ARG, "%s: NULL pointer", what);
    const int64_t across = HOW == BY_COLUMNS ? K : ceil_div(K, 128);
    QNN_REQUIRE(p.ldx >= K, QNN_ERR_INVALID_ARG, "%s: ldx below K", what);
    QNN_REQUIRE(p.ldq >= K, QNN_ERR_INVALID_ARG, "%s: ldq below K", what);
    QNN_REQUIRE(p.ld_scale >= across, QNN_ERR_INVALID_ARG, "%s: ld_scale below the number of blocks in a row", what);
    QNN_REQUIRE(aligned(p.codes, 16) && p.ldq % 16 == 0, QNN_ERR_ALIGNMENT, "%s: codes must be 16-byte aligned, ldq a multiple of 16", what);
    QNN_REQUIRE(aligned(p.scale, 16) && p.ld_scale % 16 == 0, QNN_ERR_ALIGNMENT, "%s: scales must be 16-byte aligned, ld_scale a multiple of 16", what);
    QNN_REQUIRE(aligned(p.x, (size_t)type_bytes(type)) && aligned(p.index, 8) && aligned(p.offsets, 8), QNN_ERR_ALIGNMENT,
                "%s: a pointer is not aligned to its elements", what);
    if (p.values) {
        QNN_REQUIRE(type_ok(p.values_type), QNN_ERR_INVALID_ARG, "%s: unknown type %d of the values", what, p.values_type);
        QNN_REQUIRE(p.ld_values >= K, QNN_ERR_INVALID_ARG, "%s: ld_values below K", what);
        const size_t vs = (size_t)type_bytes(p.values_type);
        QNN_REQUIRE(aligned(p.values, vs), QNN_ERR_ALIGNMENT, "%s: values are not aligned to their elements", what);
        p.vec_values = aligned(p.values, 16) && (p.ld_values * (int64_t)vs) % 16 == 0;
    }
    if (HOW == BY_COLUMNS) {
        QNN_REQUIRE(p.groups <= QNN_F8_MAX_GROUPS, QNN_ERR_UNSUPPORTED, "%s: more than %d groups", what, QNN_F8_MAX_GROUPS);
        if (p.groups == 0) return QNN_OK;
        QNN_REQUIRE(p.offsets || p.groups == 1, QNN_ERR_INVALID_ARG, "%s: offsets are NULL", what);
    }
    p.K = (int32_t)K;
    p.e5m2 = code_type == QNN_F8_E5M2;
    cudaStream_t st = as_stream(stream);
    switch (type) {
        case QNN_TYPE_F32: return launch_quant<HOW, float>(p, what, st);
        case QNN_TYPE_BF16: return launch_quant<HOW, __nv_bfloat16>(p, what, st);
        default: return launch_quant<HOW, __half>(p, what, st);
    }
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" {

int qnn_quantize_blocks_f8(const void *x, int type, int64_t rows, int64_t K, int64_t ldx, const int64_t *index, int64_t src_rows, void *codes,
                           int code_type, int64_t ldq, void *scale, int64_t ld_scale, void *values, int values_type, int64_t ld_values, void *stream)
{
    F8Source p{};
    p.x = x; p.ldx = ldx; p.rows = rows; p.index = index; p.src_rows = index ? src_rows : 0;
    p.codes = static_cast<uint8_t *>(codes); p.ldq = ldq; p.scale = static_cast<uint8_t *>(scale); p.ld_scale = ld_scale;
    p.values = values; p.values_type = values_type; p.ld_values = ld_values;
    return quant_f8<BY_ROWS>(p, type, K, code_type, "qnn_quantize_blocks_f8", stream);
}

int qnn_quantize_tiles_f8(const void *w, int type, int64_t rows, int64_t K, int64_t ldw, void *codes, int code_type, int64_t ldq, void *scale,
                          int64_t ld_scale, void *values, int values_type, int64_t ld_values, void *stream)
{
    F8Source p{};
    p.x = w; p.ldx = ldw; p.rows = rows;
    p.codes = static_cast<uint8_t *>(codes); p.ldq = ldq; p.scale = static_cast<uint8_t *>(scale); p.ld_scale = ld_scale;
    p.values = values; p.values_type = values_type; p.ld_values = ld_values;
    return quant_f8<BY_TILES>(p, type, K, code_type, "qnn_quantize_tiles_f8", stream);
}

int qnn_quantize_columns_f8(const void *x, int type, int64_t rows, int64_t K, int64_t ldx, const int64_t *offsets, int64_t groups, void *codes,
                            int code_type, int64_t ldq, void *scale, int64_t ld_scale, void *values, int values_type, int64_t ld_values, void *stream)
{
    F8Source p{};
    QNN_REQUIRE(groups <= QNN_F8_MAX_GROUPS, QNN_ERR_UNSUPPORTED, "qnn_quantize_columns_f8: more than %d groups", QNN_F8_MAX_GROUPS);
    p.x = x; p.ldx = ldx; p.rows = rows; p.offsets = offsets; p.groups = groups < 0 ? -1 : (int32_t)groups;
    p.codes = static_cast<uint8_t *>(codes); p.ldq = ldq; p.scale = static_cast<uint8_t *>(scale); p.ld_scale = ld_scale;
    p.values = values; p.values_type = values_type; p.ld_values = ld_values;
    return quant_f8<BY_COLUMNS>(p, type, K, code_type, "qnn_quantize_columns_f8", stream);
}

}  // extern "C"
