// Real values -> 8-bit floating-point codes (e4m3 or e5m2) with a power-of-two scale for each block of 128 elements of a row, 128 x 128
// of a matrix, or 128 rows of a column: the operands of the products in qnn_gemm_f8.cu.
//
// The scale is the least power of two at which the block's largest magnitude fits the codes: read off the exponent and the mantissa
// of that magnitude, so dividing by it is exact and a code is one rounding of the value (to nearest, ties to even).
//
// Every element is read once into registers, the blocks' maxima are joined across lanes (rows: 16 lanes hold a block) or through shared
// memory (tiles, columns), and codes, scales and values are written from the registers.
//
// Tiles of fp32 are bound by memory: 11008 x 4096 with bf16 values 48.7 us, 6.5 TB/s.  16-bit elements are bound by the integer pipe
// before that, and by how long loads take: 16384 rows x 2048 by index 26.1 us (pipe busy 77 %, DRAM 26 %), columns of 16384 x 4096 in
// 32 groups 71.2 us (62 %, 54 %), 5000 x 4097 in tiles, whose rows lie off 16 bytes, 41 us from cold (73 %, 16 %).
#include <type_traits>
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
    int vec_values;                              // the values' rows may be written in 16-byte pieces
    const int64_t *offsets; int32_t groups;      // columns
    int32_t log_seg, segs;                       // rows: blocks of a warp's part of a row (log2), parts a row
};

// scale byte of a block from the bits of its largest magnitude; an infinity or a NaN gives 255
template <bool E5>
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    const int e = (int)(top >> 23), low = E5 ? 15 : 8;
    const int s = e - low + ((top & 0x7fffffu) > MANT_MOST ? 1 : 0);
    return e == 255 ? 255u : s < 0 ? 0u : (uint32_t)s;
}
// 1 / scale; 0 for a scale that is NaN, whose codes are 0
__device__ __forceinline__ float scale_inverse(uint32_t s) { return s == 255u ? 0.0f : __uint_as_float((254u - s) << 23); }
__device__ __forceinline__ float scale_value(uint32_t s) { return s == 255u ? __uint_as_float(0x7fffffffu) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23); }

template <bool E5>
__device__ __forceinline__ uint32_t codes2(float lo, float hi)
{
    uint16_t r;
    if constexpr (E5) asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool E5>
__device__ __forceinline__ f32x2 decode2(uint32_t c)
{
    uint32_t h;
    if constexpr (E5) asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
    else asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
    return pair(f.x, f.y);
}

// ---- eight elements of a row, as they lie in memory --------------------------------------------------------------

// 16 lanes next to each other read 16 x 8 elements of a row.  VEC: rows start on 16 bytes.  Otherwise all of a row's pieces start at the
// same offset into 16 bytes: each lane reads the aligned unit its piece starts in, takes the next one from the next lane, and shifts the
// two into place.  A unit is read only if it holds an element of the row.  Lanes whose row is not there (row == nullptr) get zeros.
// All lanes of the warp call it.
template <typename T>
struct Eight {
    uint32_t w[2 * sizeof(T)];
};
__device__ __forceinline__ void put4(uint32_t *w, uint4 v) { w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
template <typename T>
__device__ __forceinline__ void clear_from(Eight<T> &v, int n)       // elements n, n + 1, ... become 0
{
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) {
        if constexpr (sizeof(T) == 4) v.w[i] = i < n ? v.w[i] : 0u;
        else v.w[i] = 2 * i + 1 < n ? v.w[i] : 2 * i < n ? v.w[i] & 0xffffu : 0u;
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ Eight<T> read8(const T *row, int32_t k, int32_t K)
{
    constexpr int W = 2 * (int)sizeof(T), U = W / 4;                 // words and 16-byte units of a piece
    const int left = row == nullptr ? 0 : K - k;                     // elements from here on
    Eight<T> v;
    if constexpr (VEC) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            put4(v.w + 4 * u, left > u * 16 / (int)sizeof(T) ? __ldg(reinterpret_cast<const uint4 *>(row + k) + u) : make_uint4(0, 0, 0, 0));
    } else {
        const uintptr_t at = reinterpret_cast<uintptr_t>(row + (left > 0 ? k : 0));
        const int off = (int)(at & 15);
        const uint4 *unit = reinterpret_cast<const uint4 *>(at - off);
        const int have = (16 - off) / (int)sizeof(T);                // elements of the piece in its first unit
        uint32_t x[W + 4];
#pragma unroll
        for (int u = 0; u < U; ++u)
            put4(x + 4 * u, left > (u == 0 ? 0 : have + (u - 1) * 16 / (int)sizeof(T)) ? __ldg(unit + u) : make_uint4(0, 0, 0, 0));
        // the unit after these: the next lane's first one, where that lane has read it
        const uint4 f = make_uint4(__shfl_down_sync(0xffffffffu, x[0], 1, 16), __shfl_down_sync(0xffffffffu, x[1], 1, 16),
                                   __shfl_down_sync(0xffffffffu, x[2], 1, 16), __shfl_down_sync(0xffffffffu, x[3], 1, 16));
        put4(x + W, f);
        if (((threadIdx.x & 15) == 15 || left <= 8) && left > have + (U - 1) * 16 / (int)sizeof(T) && off != 0) put4(x + W, __ldg(unit + U));
        const bool two = off & 8, one = off & 4;
#pragma unroll
        for (int i = 0; i < W + 2; ++i) x[i] = two ? x[i + 2] : x[i];
#pragma unroll
        for (int i = 0; i < W + 1; ++i) x[i] = one ? x[i + 1] : x[i];
#pragma unroll
        for (int i = 0; i < W; ++i) v.w[i] = sizeof(T) == 4 ? x[i] : __funnelshift_r(x[i], x[i + 1], 8 * (off & 2));
    }
    if (left < 8) clear_from(v, left);
    return v;
}
__device__ __forceinline__ void floats_of(const Eight<float> &v, f32x2 (&f)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pair(__uint_as_float(v.w[2 * i]), __uint_as_float(v.w[2 * i + 1]));
}
template <typename T>
__device__ __forceinline__ void floats_of(const Eight<T> &v, f32x2 (&f)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpack2(v.w[i], lo, hi, T());
        f[i] = pair(lo, hi);
    }
}
// Magnitudes: an infinity or a NaN is larger than every number, as bits are.  16-bit types are compared two at a time.
template <typename T>
__device__ __forceinline__ uint32_t mag(uint32_t w) { return w & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu); }
template <typename T>
__device__ __forceinline__ uint32_t mag_max(uint32_t a, uint32_t b)
{
    if constexpr (sizeof(T) == 4) return max(a, b);
    else return __vmaxu2(a, b);
}
// bits of the larger magnitude of a word, as fp32
__device__ __forceinline__ uint32_t mag_bits(uint32_t w, float) { return w; }
__device__ __forceinline__ uint32_t mag_bits(uint32_t w, __nv_bfloat16) { return max(w >> 16, w & 0xffffu) << 16; }
__device__ __forceinline__ uint32_t mag_bits(uint32_t w, __half) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)max(w >> 16, w & 0xffffu)))); }
template <typename T>
__device__ __forceinline__ uint32_t mag8(const Eight<T> &v)
{
    uint32_t t = mag<T>(v.w[0]);
#pragma unroll
    for (int i = 1; i < 2 * (int)sizeof(T); ++i) t = mag_max<T>(t, mag<T>(v.w[i]));
    return t;
}

// ---- what the codes stand for ------------------------------------------------------------------------------------

// Eight values of a row from k on: 16 lanes next to each other hold 16 x 8, all lanes of the warp call it (`on`: those with a row).
// Where rows do not start on 16 bytes, each lane writes the aligned unit that its piece starts in, with the end of the lane's before;
// the ends of the 128 go element by element.
template <typename V>
__device__ __forceinline__ void put_values(V *row, int32_t k, int32_t K, const f32x2 (&f)[4], bool vec, bool on)
{
    constexpr int W = 2 * (int)sizeof(V), U = W / 4, PER = 16 / (int)sizeof(V);       // words, units; elements of a unit
    uint32_t w[W];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpair(f[i], lo, hi);
        if constexpr (sizeof(V) == 4) { w[2 * i] = __float_as_uint(lo); w[2 * i + 1] = __float_as_uint(hi); }
        else w[i] = pack2(lo, hi, V());
    }
    const int left = on ? K - k : 0;
    V *at = row + (on ? k : 0);
    if (vec) {                                                       // (uniform)
        if (left >= 8) {
#pragma unroll
            for (int u = 0; u < U; ++u) *(reinterpret_cast<uint4 *>(at) + u) = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) {
                if constexpr (sizeof(V) == 4) reinterpret_cast<uint32_t *>(at)[i] = w[i];
                else reinterpret_cast<uint16_t *>(at)[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
            }
        return;
    }
    const int off = (int)(reinterpret_cast<uintptr_t>(at) & 15), behind = off / (int)sizeof(V), lane16 = threadIdx.x & 15;
    // x: the last unit of the lane's before, then this lane's; t: the same moved so that t[4 + i] starts at word i of the first unit
    uint32_t x[W + 4], t[W + 4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __shfl_up_sync(0xffffffffu, w[W - 4 + i], 1, 16);
#pragma unroll
    for (int i = 0; i < W; ++i) x[4 + i] = w[i];
#pragma unroll
    for (int i = W + 3; i >= 2; --i) x[i] = off & 8 ? x[i - 2] : x[i];
#pragma unroll
    for (int i = W + 3; i >= 3; --i) t[i] = off & 4 ? x[i - 1] : x[i];
    bool whole[U];                                                   // all elements of the unit are this lane's or the one's before
#pragma unroll
    for (int u = 0; u < U; ++u) {
        whole[u] = left > 0 && (u + 1) * PER - behind <= left && (u > 0 || behind == 0 || lane16 > 0);
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = sizeof(V) == 2 && (off & 2) ? __funnelshift_r(t[3 + 4 * u + i], t[4 + 4 * u + i], 16) : t[4 + 4 * u + i];
        if (whole[u]) *reinterpret_cast<uint4 *>(at - behind + u * PER) = make_uint4(y[0], y[1], y[2], y[3]);
    }
    const bool next_whole = lane16 < 15 && PER - behind <= left - 8; // the next lane's first unit, which holds this lane's last elements
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int u = (i + behind) / PER;
        if (i < left && !(u == 0 ? whole[0] : u < U ? whole[U - 1] : next_whole)) {
            if constexpr (sizeof(V) == 4) reinterpret_cast<uint32_t *>(at)[i] = w[i];
            else reinterpret_cast<uint16_t *>(at)[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
        }
    }
}
// The values' type as an argument of f: one copy of its code for each, one branch a thread.
struct Nothing {};
template <typename F>
__device__ __forceinline__ void with_values(const F8Source &p, F f)
{
    if (p.values == nullptr) f(Nothing());
    else if (p.values_type == QNN_TYPE_F32) f(float());
    else if (p.values_type == QNN_TYPE_BF16) f(__nv_bfloat16());
    else f(__half());
}
template <bool E5>
__device__ __forceinline__ uint2 encode8(const f32x2 (&f)[4], const f32x2 (&inv)[4])
{
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpair(mul2(f[i], inv[i]), lo, hi);
        c[i] = codes2<E5>(lo, hi);
    }
    return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}
template <bool E5>
__device__ __forceinline__ void decode8(uint2 q, const f32x2 (&scale)[4], f32x2 (&f)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = mul2(decode2<E5>((i < 2 ? q.x : q.y) >> (16 * (i & 1))), scale[i]);
}

// ---- 1024 elements of a row: four times 256, a warp's lanes next to each other ------------------------------------

// words A and following of x, moved down by another `bits` (0 or 16)
template <typename T, int A>
__device__ __forceinline__ void shift_down(const uint32_t *x, int bits, Eight<T> &v)
{
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) v.w[i] = sizeof(T) == 4 ? x[i + A] : __funnelshift_r(x[i + A], x[i + A + 1], bits);
}
// As read8, k the first of this lane's elements; the offset into 16 bytes is the warp's.
template <typename T, bool VEC>
__device__ __forceinline__ void read_segment(const T *row, int32_t k, int32_t K, Eight<T> (&v)[4])
{
    constexpr int W = 2 * (int)sizeof(T), U = W / 4, PER = 16 / (int)sizeof(T);
    const int left = row == nullptr ? 0 : K - k, lane = threadIdx.x & 31;
    if constexpr (VEC) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < U; ++i)
                put4(v[u].w + 4 * i, left > 256 * u + i * PER ? __ldg(reinterpret_cast<const uint4 *>(row + k + 256 * u) + i) : make_uint4(0, 0, 0, 0));
    } else {
        const int off = (int)(reinterpret_cast<uintptr_t>(row) & 15), have = (16 - off) / (int)sizeof(T);
        const T *at = row + (row == nullptr ? 0 : k - off / (int)sizeof(T));       // (16-byte aligned)
        uint32_t x[4][W + 4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < U; ++i)
                put4(x[u] + 4 * i, left > 256 * u + (i == 0 ? 0 : have + (i - 1) * PER) ? __ldg(reinterpret_cast<const uint4 *>(at + 256 * u) + i) : make_uint4(0, 0, 0, 0));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            // the unit after these: the next lane's first one, or the first lane's of the next 256
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t next = __shfl_down_sync(0xffffffffu, x[u][i], 1), first = u < 3 ? __shfl_sync(0xffffffffu, x[u < 3 ? u + 1 : 3][i], 0) : 0u;
                x[u][W + i] = lane == 31 ? first : next;
            }
            const int l = left - 256 * u;
            if (((lane == 31 && u == 3) || l <= 8) && l > have + (U - 1) * PER && off != 0) put4(x[u] + W, __ldg(reinterpret_cast<const uint4 *>(at + 256 * u) + U));
        }
        const int bits = 8 * (off & 2);
        switch (off >> 2) {
            case 0:
#pragma unroll
                for (int u = 0; u < 4; ++u) shift_down<T, 0>(x[u], bits, v[u]);
                break;
            case 1:
#pragma unroll
                for (int u = 0; u < 4; ++u) shift_down<T, 1>(x[u], bits, v[u]);
                break;
            case 2:
#pragma unroll
                for (int u = 0; u < 4; ++u) shift_down<T, 2>(x[u], bits, v[u]);
                break;
            default:
#pragma unroll
                for (int u = 0; u < 4; ++u) shift_down<T, 3>(x[u], bits, v[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (left < 256 * u + 8) clear_from(v[u], left - 256 * u);
}

template <typename V, int A>
__device__ __forceinline__ void store_shifted(const uint32_t *x, bool half, V *unit, const bool *whole)
{
    constexpr int U = (int)sizeof(V) / 2;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            y[i] = sizeof(V) == 2 ? (half ? __funnelshift_r(A + 1 <= 4 + 4 * u + i ? x[3 + 4 * u + i - A] : 0u, x[4 + 4 * u + i - A], 16) : x[4 + 4 * u + i - A]) : x[4 + 4 * u + i - A];
        if (whole[u]) *reinterpret_cast<uint4 *>(unit + u * (16 / (int)sizeof(V))) = make_uint4(y[0], y[1], y[2], y[3]);
    }
}
// Part u of a row's 1024 values (rows that do not start on 16 bytes): as put_values, the unit that a lane's piece starts in holds the end of
// the lane's before, or (first lane) of the last lane's of the part before, which `carry` hands on.  row: not null where left > 0.
template <typename V>
__device__ __forceinline__ void put_part(V *row, int32_t k, int32_t K, const f32x2 (&f)[4], int u4, uint32_t (&carry)[4])
{
    constexpr int W = 2 * (int)sizeof(V), U = W / 4, PER = 16 / (int)sizeof(V);
    const int lane = threadIdx.x & 31, left = K - k;
    uint32_t x[W + 4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpair(f[i], lo, hi);
        if constexpr (sizeof(V) == 4) { x[4 + 2 * i] = __float_as_uint(lo); x[5 + 2 * i] = __float_as_uint(hi); }
        else x[4 + i] = pack2(lo, hi, V());
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t before = __shfl_up_sync(0xffffffffu, x[W + i], 1);
        x[i] = lane == 0 ? carry[i] : before;
        carry[i] = __shfl_sync(0xffffffffu, x[W + i], 31);
    }
    const int off = (int)(reinterpret_cast<uintptr_t>(row) & 15), behind = off / (int)sizeof(V);
    V *at = row + k;
    bool whole[U];
#pragma unroll
    for (int u = 0; u < U; ++u) whole[u] = left > 0 && (u + 1) * PER - behind <= left && (u > 0 || behind == 0 || lane > 0 || u4 > 0);
    const bool half = off & 2;
    switch (off >> 2) {                                  // (the warp's)
        case 0: store_shifted<V, 0>(x, half, at - behind, whole); break;
        case 1: store_shifted<V, 1>(x, half, at - behind, whole); break;
        case 2: store_shifted<V, 2>(x, half, at - behind, whole); break;
        default: store_shifted<V, 3>(x, half, at - behind, whole);
    }
    // the ends: before the first whole unit of the 1024, behind the last one, and where the row ends
    if (u4 == 0 || u4 == 3 || __any_sync(0xffffffffu, left < 24)) {
        const bool next_whole = (lane < 31 || u4 < 3) && PER - behind <= left - 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int u = (i + behind) / PER;
            if (i < left && !(u == 0 ? whole[0] : u < U ? whole[U - 1] : next_whole)) {
                if constexpr (sizeof(V) == 4) reinterpret_cast<uint32_t *>(at)[i] = x[4 + i];
                else reinterpret_cast<uint16_t *>(at)[i] = (uint16_t)(x[4 + i / 2] >> (16 * (i & 1)));
            }
        }
    }
}

// ---- blocks of a row ---------------------------------------------------------------------------------------------

// 16 lanes hold a block, eight elements each; a warp takes eight blocks, 2^log_seg next to each other of each of 8 / 2^log_seg rows (WIDE:
// all eight of one row), four in flight a lane.
template <typename T, bool VEC, bool WIDE, bool E5>
__global__ void __launch_bounds__(128)
quant_rows_f8_kernel(const F8Source p)
{
    const int lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
    const uint32_t warp = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const uint32_t rg = warp / (uint32_t)p.segs;
    const int32_t seg = (int32_t)(warp - rg * (uint32_t)p.segs);
    const int log_seg = WIDE ? 3 : p.log_seg;
    const int64_t row0 = (int64_t)rg << (3 - log_seg);
    const int32_t K16 = (p.K + 15) & ~15;
    auto row_of = [&](int u) { return WIDE ? row0 : row0 + ((2 * u + half) >> log_seg); };
    auto blk_of = [&](int u) { return (seg << log_seg) + ((2 * u + half) & ((1 << log_seg) - 1)); };
    auto source = [&](int64_t row) -> const T * {
        if (row >= p.rows) return nullptr;
        int64_t from = row;
        if (p.index) {
            from = __ldg(p.index + row);
            if (from < 0 || from >= p.src_rows) return nullptr;
        }
        return static_cast<const T *>(p.x) + from * p.ldx;
    };
    griddep_wait();
    Eight<T> v[4];
    const int32_t k0 = (seg << 10) + 8 * lane;           // (WIDE)
    if constexpr (WIDE) {
        read_segment<T, VEC>(source(row0), k0, p.K, v);
    } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = read8<T, VEC>(source(row_of(u)), (blk_of(u) << 7) + 8 * l16, p.K);
    }
    griddep_launch_dependents();
    const bool chained = WIDE && !p.vec_values;
    auto encode = [&](auto kind) {                       // V: the values' type; nothing: none
        using V = decltype(kind);
        constexpr bool VALUES = !std::is_same<V, Nothing>::value;
        uint32_t carry[4] = {0u, 0u, 0u, 0u};
        [[maybe_unused]] uint8_t *codes = p.codes + row0 * p.ldq + k0, *scale = p.scale + row0 * p.ld_scale + 8 * seg + half;  // (WIDE)
        V *values = static_cast<V *>(p.values) + (VALUES ? row0 * p.ld_values : 0);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t row = row_of(u);
            const int32_t k = WIDE ? k0 + 256 * u : (blk_of(u) << 7) + 8 * l16;
            if (WIDE && (seg << 10) + 256 * u >= p.K) break;         // (the warp's)
            uint32_t top = mag8(v[u]);
#pragma unroll
            for (int d = 8; d > 0; d /= 2) top = mag_max<T>(top, __shfl_xor_sync(0xffffffffu, top, d));
            const uint32_t s = scale_byte<E5>(mag_bits(top, T()));
            f32x2 f[4], by[4];
            floats_of(v[u], f);
            const float inv = scale_inverse(s), val = scale_value(s);
#pragma unroll
            for (int i = 0; i < 4; ++i) by[i] = pair(inv, inv);
            uint2 q = encode8<E5>(f, by);
            if (s == 255u) q = make_uint2(0u, 0u);                   // (0 times an infinity is a NaN)
            const bool there = row < p.rows && k < K16;
            if (there) {
                if constexpr (WIDE) {
                    *reinterpret_cast<uint2 *>(codes + 256 * u) = q;
                    if (l16 == 0) scale[2 * u] = (uint8_t)s;
                } else {
                    *reinterpret_cast<uint2 *>(p.codes + row * p.ldq + k) = q;
                    if (l16 == 0) p.scale[row * p.ld_scale + blk_of(u)] = (uint8_t)s;
                }
            }
            if constexpr (VALUES) {
#pragma unroll
                for (int i = 0; i < 4; ++i) by[i] = pair(val, val);
                decode8<E5>(q, by, f);
                if (chained) put_part(values, k, row < p.rows ? p.K : 0, f, u, carry);           // (no row: nothing left of it)
                else put_values(WIDE ? values : static_cast<V *>(p.values) + row * p.ld_values, k, p.K, f, p.vec_values != 0, there && k < p.K);
            }
        }
    };
    with_values(p, encode);
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

// 128 rows x 128 columns: 16 lanes hold a row's 128 columns, eight each, and a thread every sixteenth row.  Elements stay as they
// lie in memory until they are encoded, so that four blocks (of 16-bit types) fit an SM: one's loads go on while the others join and write.
template <typename T, bool VEC, bool COLUMNS, bool E5>
__global__ void __launch_bounds__(TILE_THREADS, sizeof(T) == 4 ? 2 : 4)
quant_tiles_f8_kernel(const F8Source p)
{
    constexpr int W = 2 * (int)sizeof(T);
    __shared__ uint4 tops[8][8 * sizeof(T)];             // of 128 columns, a row a warp
    __shared__ __align__(8) uint8_t bytes[128];
    __shared__ int64_t where[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, l16 = tid & 15, r16 = tid >> 4;
    const int32_t blk = blockIdx.y, tile = blockIdx.x;
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
    const int32_t k = tile * 128 + 8 * l16;
    Eight<T> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i * 16 + r16;
        v[i] = read8<T, VEC>(r < rows ? src + (int64_t)r * p.ldx : nullptr, k, p.K);
    }
    griddep_launch_dependents();
    uint32_t s8[2];                                  // this thread's columns' scale bytes
    if (COLUMNS) {
        uint32_t m[W];
#pragma unroll
        for (int c = 0; c < W; ++c) {
            uint32_t t = mag<T>(v[0].w[c]);
#pragma unroll
            for (int i = 1; i < 8; ++i) t = mag_max<T>(t, mag<T>(v[i].w[c]));
            m[c] = mag_max<T>(t, __shfl_xor_sync(0xffffffffu, t, 16));
        }
        if (lane < 16)
#pragma unroll
            for (int u = 0; u < W / 4; ++u) tops[warp][l16 * (W / 4) + u] = make_uint4(m[4 * u], m[4 * u + 1], m[4 * u + 2], m[4 * u + 3]);
        __syncthreads();
        if (tid < 128) {
            uint32_t t = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                if constexpr (sizeof(T) == 4) t = max(t, reinterpret_cast<const uint32_t *>(tops[w])[tid]);
                else t = max(t, (uint32_t)reinterpret_cast<const uint16_t *>(tops[w])[tid]);
            }
            const uint32_t b = scale_byte<E5>(mag_bits(t, T()));
            bytes[tid] = (uint8_t)b;
            if (tile * 128 + tid < p.K) p.scale[(int64_t)blk * p.ld_scale + tile * 128 + tid] = (uint8_t)b;
        }
        __syncthreads();
        const uint2 b8 = *reinterpret_cast<const uint2 *>(&bytes[8 * l16]);
        s8[0] = b8.x; s8[1] = b8.y;
    } else {
        uint32_t t = mag8(v[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) t = mag_max<T>(t, mag8(v[i]));
        t = __reduce_max_sync(0xffffffffu, mag_bits(t, T()));
        uint32_t *part = reinterpret_cast<uint32_t *>(tops[0]);
        if (lane == 0) part[warp] = t;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) t = max(t, part[w]);
        const uint32_t b = scale_byte<E5>(t);
        if (tid == 0) p.scale[(int64_t)blk * p.ld_scale + tile] = (uint8_t)b;
        s8[0] = s8[1] = b * 0x01010101u;
    }
    f32x2 inv[4], val[4];
    uint2 keep = make_uint2(0u, 0u);                 // codes of columns with a NaN scale are 0
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint32_t a = s8[c / 2] >> (16 * (c & 1)) & 0xffu, b = s8[c / 2] >> (16 * (c & 1) + 8) & 0xffu;
        inv[c] = pair(scale_inverse(a), scale_inverse(b));
        val[c] = pair(scale_value(a), scale_value(b));
        const uint32_t both = ((a != 255u ? 0xffu : 0u) | (b != 255u ? 0xff00u : 0u)) << (16 * (c & 1));
        if (c < 2) keep.x |= both;
        else keep.y |= both;
    }
    // (columns: the rows that fill a group up to whole blocks are written too, as zeros)
    auto encode = [&](auto kind) {
        using V = decltype(kind);
        constexpr bool VALUES = !std::is_same<V, Nothing>::value;
        const int64_t out0 = (int64_t)blk * 128 + r16;
        uint8_t *codes = p.codes + out0 * p.ldq + k;
        V *values = static_cast<V *>(p.values) + (VALUES ? out0 * p.ld_values : 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool there = (COLUMNS || i * 16 + r16 < rows) && k < K16;
            f32x2 f[4];
            floats_of(v[i], f);
            uint2 q = encode8<E5>(f, inv);
            q.x &= keep.x; q.y &= keep.y;
            if (there) *reinterpret_cast<uint2 *>(codes) = q;
            codes += 16 * p.ldq;
            if constexpr (VALUES) {
                decode8<E5>(q, val, f);
                put_values(values, k, p.K, f, p.vec_values != 0, there && k < p.K);
                values += 16 * p.ld_values;
            }
        }
    };
    with_values(p, encode);
}

// ---- host --------------------------------------------------------------------------------------------------------

enum { BY_ROWS, BY_TILES, BY_COLUMNS };

template <int HOW, typename T, bool E5>
int launch_quant(F8Source p, const char *what, cudaStream_t st)
{
    const bool vec = aligned(p.x, 16) && (p.ldx * (int64_t)sizeof(T)) % 16 == 0;
    const int64_t nblk = ceil_div(p.K, 128);
    if (HOW == BY_ROWS) {
        p.log_seg = nblk > 2 ? 3 : nblk > 1 ? 1 : 0;
        p.segs = (int32_t)ceil_div(nblk, 1 << p.log_seg);
        const int64_t warps = ceil_div(p.rows, 8 >> p.log_seg) * p.segs;
        QNN_REQUIRE(warps < ((int64_t)1 << 32) - 4, QNN_ERR_UNSUPPORTED, "%s: too many blocks", what);
        const dim3 grid((unsigned)ceil_div(warps, 4)), block(128);
        if (p.log_seg == 3) {
            if (vec) QNN_CUDA(launch_pdl(quant_rows_f8_kernel<T, true, true, E5>, grid, block, 0, st, p));
            else QNN_CUDA(launch_pdl(quant_rows_f8_kernel<T, false, true, E5>, grid, block, 0, st, p));
        } else {
            if (vec) QNN_CUDA(launch_pdl(quant_rows_f8_kernel<T, true, false, E5>, grid, block, 0, st, p));
            else QNN_CUDA(launch_pdl(quant_rows_f8_kernel<T, false, false, E5>, grid, block, 0, st, p));
        }
    } else {
        const int64_t blocks = HOW == BY_COLUMNS ? p.rows / 128 + p.groups : ceil_div(p.rows, 128);
        QNN_REQUIRE(blocks < 65536, QNN_ERR_UNSUPPORTED, "%s: 65536 blocks of 128 rows and more", what);
        const dim3 grid((unsigned)nblk, (unsigned)blocks);
        if (vec) QNN_CUDA(launch_pdl(quant_tiles_f8_kernel<T, true, HOW == BY_COLUMNS, E5>, grid, dim3(TILE_THREADS), 0, st, p));
        else QNN_CUDA(launch_pdl(quant_tiles_f8_kernel<T, false, HOW == BY_COLUMNS, E5>, grid, dim3(TILE_THREADS), 0, st, p));
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
    const bool e5 = code_type == QNN_F8_E5M2;
    cudaStream_t st = as_stream(stream);
    switch (type) {
        case QNN_TYPE_F32: return e5 ? launch_quant<HOW, float, true>(p, what, st) : launch_quant<HOW, float, false>(p, what, st);
        case QNN_TYPE_BF16: return e5 ? launch_quant<HOW, __nv_bfloat16, true>(p, what, st) : launch_quant<HOW, __nv_bfloat16, false>(p, what, st);
        default: return e5 ? launch_quant<HOW, __half, true>(p, what, st) : launch_quant<HOW, __half, false>(p, what, st);
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
