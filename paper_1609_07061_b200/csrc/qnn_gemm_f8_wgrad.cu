// Weight gradients of groups of rows from 8-bit floating-point codes: dw[g][n,k] = sum over the group's rows m of DY[m,n] X[m,k].
//
// Both operands carry one scale for each column of a block of 128 rows, so the sum over a block is a plain product of codes, taken to
// its place by 2^(sy[n] + sx[k] - 254): sums of blocks and of the group are held in fp32.  A code of either type is an fp16 number
// exactly (inf and NaN too) and a product of two is exact in fp32, so the codes are multiplied as fp16.
//
// One CTA owns 128 x 128 results of a group; sixteen warps own 32 x 32 of them each.  Rows go through shared memory 64 at a time, the next
// 64 on their way in registers meanwhile, and are turned round by transposing matrix loads.  Every load is a plain one of 16 bytes
// within a row, and only blocks of the group itself are read: buffers need hold no more than the groups' blocks.
// 16384 rows over 32 groups, 4096 x 2048 (e5m2): 2159 us, 127 TFLOP/s; 4096 x 4096 x 4096 in one group 700 us, 196 TFLOP/s.  Far from
// its floor (98 and 41 us).  At 4096 rows, 8 groups, 2048 x 2048 the tensor pipe is busy 26 % of the time, the integer pipe 23 %; warps
// wait most for the queue of loads and stores (scales come a byte at a time, results leave one by one), then for shared memory.
// Conversions are not what bounds it: e5m2 by the conversion instruction takes 2203 instead of 2149.  Eight warps of 64 x 32, which
// read shared memory less often, take 2547.
#include <cuda_fp8.h>
#include "qnn_f8.cuh"

namespace qnn {
namespace {

constexpr int WG_T = 128, WG_ROWS = 64, WG_THREADS = 512;
constexpr int WG_PITCH = WG_T + 8;                   // halves; eight rows of 16 bytes then lie in different banks
constexpr int WG_BYTES = 2 * 2 * WG_ROWS * WG_PITCH * 2;

// two codes as halves: an e5m2 code is the upper byte of its fp16 number
template <int TYPE>
__device__ __forceinline__ uint32_t low_halves(uint32_t codes)
{
    if constexpr (TYPE == QNN_F8_E5M2) return __byte_perm(codes, 0u, 0x1404);
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes & 0xffffu), __NV_E4M3);
    return (uint32_t)h.x | (uint32_t)h.y << 16;
}
template <int TYPE>
__device__ __forceinline__ uint32_t high_halves(uint32_t codes)
{
    if constexpr (TYPE == QNN_F8_E5M2) return __byte_perm(codes, 0u, 0x3424);
    return low_halves<TYPE>(codes >> 16);
}
// 16 codes as 16 halves
template <int TYPE>
__device__ __forceinline__ void put_codes(__half *to, uint4 v)
{
    uint4 *d = reinterpret_cast<uint4 *>(to);
    d[0] = make_uint4(low_halves<TYPE>(v.x), high_halves<TYPE>(v.x), low_halves<TYPE>(v.y), high_halves<TYPE>(v.y));
    d[1] = make_uint4(low_halves<TYPE>(v.z), high_halves<TYPE>(v.z), low_halves<TYPE>(v.w), high_halves<TYPE>(v.w));
}
__device__ __forceinline__ void load_trans(uint32_t (&r)[4], const __half *at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"((uint32_t)__cvta_generic_to_shared(at)) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// v 2^(s + t - 254), in two steps: the whole power need not be an fp32 number, its halves are normal ones.  Below 2^-252 any sum of a
// block (at most 128 57344^2 < 2^39) is zero in fp32 either way.
__device__ __forceinline__ float scaled(float v, int s, int t)
{
    const int e = s + t - 254 > -252 ? s + t - 254 : -252, h = e >> 1;
    const float r = v * __int_as_float((h + 127) << 23) * __int_as_float((e - h + 127) << 23);
    return s == 255 || t == 255 ? __int_as_float(0x7fffffff) : r;
}

template <typename TOUT, int DY, int X>
__global__ void __launch_bounds__(WG_THREADS) wgrad_f8_kernel(const WgParams p)
{
    extern __shared__ __align__(16) uint8_t wg_smem[];
    typedef __half Buffer[WG_ROWS][WG_PITCH];
    Buffer *sy = reinterpret_cast<Buffer *>(wg_smem), *sx = sy + 2;
    __shared__ int32_t where[2];                     // the group's first block and its number of blocks
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t tile = (int32_t)blockIdx.x, per = p.tiles_n * p.tiles_k;
    const int32_t g = tile / per, tn = (tile - g * per) / p.tiles_k, tk = tile - g * per - tn * p.tiles_k;
    if (warp == 0) {
        // offsets held to rise and to stay in 0..M, as the quantiser holds them
        int32_t carry = 0, blocks = 0, len = (int32_t)p.M;
        for (int32_t i0 = 0; p.offsets && i0 <= g + 1; i0 += 32) {
            const int32_t i = i0 + lane;
            int64_t o = i <= g + 1 ? __ldg(p.offsets + i) : 0;
            o = o < 0 ? 0 : o > p.M ? p.M : o;
            int32_t s = (int32_t)o > carry ? (int32_t)o : carry;
            for (int d = 1; d < 32; d *= 2) {
                const int32_t u = __shfl_up_sync(0xffffffffu, s, d);
                if (lane >= d && u > s) s = u;
            }
            const int32_t up = __shfl_up_sync(0xffffffffu, s, 1), before = lane == 0 ? carry : up;
            int32_t b = i >= 1 && i <= g ? (s - before + 127) / 128 : 0;
            for (int d = 16; d > 0; d /= 2) b += __shfl_xor_sync(0xffffffffu, b, d);
            blocks += b;
            if (g + 1 - i0 < 32) len = __shfl_sync(0xffffffffu, s - before, g + 1 - i0);
            carry = __shfl_sync(0xffffffffu, s, 31);
        }
        if (lane == 0) { where[0] = blocks; where[1] = (len + 127) / 128; }
    }
    __syncthreads();
    const int32_t blk0 = where[0], steps = where[1] * (128 / WG_ROWS);

    // a thread's 16 bytes of 64 rows x 128 columns
    const int row = tid >> 3, col = (tid & 7) * 16;
    const bool has_y = tn * WG_T + col < p.N, has_x = tk * WG_T + col < p.K;
    const uint8_t *py = p.dy + ((int64_t)blk0 * 128 + row) * p.ld_dy + tn * WG_T + col;
    const uint8_t *px = p.x + ((int64_t)blk0 * 128 + row) * p.ldx + tk * WG_T + col;
    const uint4 none = make_uint4(0, 0, 0, 0);
    auto fetch = [&](int32_t s, uint4 &a, uint4 &b) {
        a = has_y ? __ldg(reinterpret_cast<const uint4 *>(py + (int64_t)s * WG_ROWS * p.ld_dy)) : none;
        b = has_x ? __ldg(reinterpret_cast<const uint4 *>(px + (int64_t)s * WG_ROWS * p.ldx)) : none;
    };
    const int wn = (warp >> 2) * 32, wk = (warp & 3) * 32, fr = lane >> 2, fc = 2 * (lane & 3);
    float sum[2][4][4] = {}, part[2][4][4] = {};
    uint4 a, b;
    if (steps > 0) fetch(0, a, b);
    for (int32_t s = 0; s < steps; ++s) {
        const int h = s & 1;
        put_codes<DY>(&sy[h][row][col], a);
        put_codes<X>(&sx[h][row][col], b);
        __syncthreads();                             // (two buffers: a warp here has left the one before last)
        if (s + 1 < steps) fetch(s + 1, a, b);
#pragma unroll
        for (int k0 = 0; k0 < WG_ROWS; k0 += 16) {
            uint32_t fa[2][4], fb[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) load_trans(fa[i], &sy[h][k0 + (lane >> 4) * 8 + (lane & 7)][wn + 16 * i + (lane >> 3 & 1) * 8]);
#pragma unroll
            for (int j = 0; j < 2; ++j) load_trans(fb[j], &sx[h][k0 + (lane >> 3 & 1) * 8 + (lane & 7)][wk + 16 * j + (lane >> 4) * 8]);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) mma_f16(part[i][j], fa[i], fb[j >> 1][2 * (j & 1)], fb[j >> 1][2 * (j & 1) + 1]);
        }
        if ((s & 1) == 0) continue;
        const int64_t blk = blk0 + (s >> 1);
        // scales as fp32 numbers 2^(s - 127), by their bits (0 and infinity: scales 0 and 255, which take the other way)
        float ey[2][2], ex[4][2];
        float y0 = 1.0f, y1 = 1.0f, x0 = 1.0f, x1 = 1.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int32_t k = tk * WG_T + wk + 8 * i + fc + u;
                ex[i][u] = __int_as_float((k < p.K ? (int)p.x_scale[blk * p.ld_xs + k] : 127) << 23);
                x0 = fminf(x0, ex[i][u]); x1 = fmaxf(x1, ex[i][u]);
                if (i < 2) {
                    const int32_t n = tn * WG_T + wn + 16 * i + 8 * u + fr;
                    ey[i][u] = __int_as_float((n < p.N ? (int)p.dy_scale[blk * p.ld_dys + n] : 127) << 23);
                    y0 = fminf(y0, ey[i][u]); y1 = fmaxf(y1, ey[i][u]);
                }
            }
        // Where every product of two scales is a normal number it is exact: a multiplication and a multiply-add a result, which leave the
        // integer pipe to the conversions of codes.
        const float low = y0 * x0, high = y1 * x1;
        if (__all_sync(0xffffffffu, y0 > 0.0f && x0 > 0.0f && low >= 1.17549435e-38f && high <= 3.40282347e38f)) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[i][j][e] = fmaf(part[i][j][e], ey[i][e >> 1] * ex[j][e & 1], sum[i][j][e]);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        sum[i][j][e] += scaled(part[i][j][e], __float_as_int(ey[i][e >> 1]) >> 23, __float_as_int(ex[j][e & 1]) >> 23);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[i][j][e] = 0.0f;
    }
    TOUT *dw = static_cast<TOUT *>(p.dw);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t n = tn * WG_T + wn + 16 * i + 8 * (e >> 1) + fr, k = tk * WG_T + wk + 8 * j + fc + (e & 1);
                if (n < p.N && k < p.K) from_float(sum[i][j][e], dw[((int64_t)g * p.N + n) * p.ld_dw + k]);
            }
}

template <typename TOUT, int DY, int X>
int launch_wgrad(const char *what, const WgParams &p, unsigned grid, cudaStream_t st)
{
    static std::atomic<bool> done[64];
    auto kern = wgrad_f8_kernel<TOUT, DY, X>;
    if (int rc = opt_in(kern, WG_BYTES, done)) return rc;
    profile_before(st);
    kern<<<grid, WG_THREADS, WG_BYTES, st>>>(p);
    profile_after(st);
    return check_launch(what);
}

}  // namespace

int run_f8_wgrad(const char *what, WgParams p, int dy_type, int x_type, int out_type, cudaStream_t st)
{
    p.tiles_n = (int32_t)ceil_div(p.N, WG_T); p.tiles_k = (int32_t)ceil_div(p.K, WG_T);
    const int64_t tiles = (int64_t)p.tiles_n * p.tiles_k;
    QNN_REQUIRE(tiles < (int64_t)1 << 28 && tiles * p.groups < (int64_t)1 << 30, QNN_ERR_UNSUPPORTED, "%s: too many output tiles", what);
    const unsigned grid = (unsigned)(tiles * p.groups);
    const bool e4 = dy_type == QNN_F8_E4M3, f4 = x_type == QNN_F8_E4M3;
    auto typed = [&](auto out) {
        typedef decltype(out) T;
        return e4 ? (f4 ? launch_wgrad<T, QNN_F8_E4M3, QNN_F8_E4M3>(what, p, grid, st) : launch_wgrad<T, QNN_F8_E4M3, QNN_F8_E5M2>(what, p, grid, st))
                  : (f4 ? launch_wgrad<T, QNN_F8_E5M2, QNN_F8_E4M3>(what, p, grid, st) : launch_wgrad<T, QNN_F8_E5M2, QNN_F8_E5M2>(what, p, grid, st));
    };
    return out_type == QNN_TYPE_F32 ? typed(float()) : out_type == QNN_TYPE_BF16 ? typed(__nv_bfloat16()) : typed(__half());
}

}  // namespace qnn
