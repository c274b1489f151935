// Element types of the operators that take real tensors in 32 or 16 bits (QNN_TYPE_*): loads of W consecutive elements
// as fp32, stores of W fp32 values rounded once to the type.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "qnn_internal.cuh"

namespace qnn {

inline bool type_ok(int type) { return type == QNN_TYPE_F32 || type == QNN_TYPE_BF16 || type == QNN_TYPE_F16; }
inline int64_t type_bytes(int type) { return type == QNN_TYPE_F32 ? 4 : 2; }

#ifdef __CUDACC__
template <int TYPE> struct ElemOf;
template <> struct ElemOf<QNN_TYPE_F32> { using T = float; };
template <> struct ElemOf<QNN_TYPE_BF16> { using T = __nv_bfloat16; };
template <> struct ElemOf<QNN_TYPE_F16> { using T = __half; };

__device__ __forceinline__ float bits_to_float(uint32_t half_bits, __nv_bfloat16) { return __uint_as_float(half_bits << 16); }
__device__ __forceinline__ float bits_to_float(uint32_t half_bits, __half) { return __half2float(__ushort_as_half((unsigned short)half_bits)); }

// two 16-bit elements of a 32-bit word
__device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi, __nv_bfloat16)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    lo = f.x; hi = f.y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_float(float x, float &o) { o = x; }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16 &o) { o = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_float(float x, __half &o) { o = __float2half_rn(x); }

// Two fp32 values in one 64-bit register pair: sm_100 adds, multiplies and fuses pairs with one instruction, which halves
// the issue slots of the element loops.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float lo, float hi)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(f32x2 v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) { f32x2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
// maximum that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// W consecutive elements in registers as they lie in memory.  W = 8 is one or two 16-byte accesses, W = 2 one access of
// a pair, W = 1 a single element; the address must be a multiple of min(16, W * sizeof(T)) bytes.
template <typename T, int W>
struct Piece {
    T e[W];
    __device__ __forceinline__ float get(int i) const { return to_float(e[i]); }
};
template <typename T>
struct Piece<T, 8> {
    uint32_t w[sizeof(T) * 2];
};

template <typename T, int W>
__device__ __forceinline__ void load_piece(const T *p, Piece<T, W> &v)
{
    if constexpr (W == 8) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        v.w[0] = a.x; v.w[1] = a.y; v.w[2] = a.z; v.w[3] = a.w;
        if constexpr (sizeof(T) == 4) {
            const uint4 b = *(reinterpret_cast<const uint4 *>(p) + 1);
            v.w[4] = b.x; v.w[5] = b.y; v.w[6] = b.z; v.w[7] = b.w;
        }
    } else if constexpr (W == 2) {
        if constexpr (sizeof(T) == 4) {
            const float2 a = *reinterpret_cast<const float2 *>(p);
            v.e[0] = a.x; v.e[1] = a.y;
        } else {
            *reinterpret_cast<uint32_t *>(v.e) = *reinterpret_cast<const uint32_t *>(p);
        }
    } else {
        v.e[0] = *p;
    }
}
template <typename T, int W>
__device__ __forceinline__ void piece_to_floats(const Piece<T, W> &v, float (&f)[W])
{
    if constexpr (W == 8) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v.w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) unpack2(v.w[i], f[2 * i], f[2 * i + 1], T());
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) f[i] = to_float(v.e[i]);
    }
}
// W fp32 values, each rounded once, to W consecutive elements (alignment as for load_piece)
template <typename T, int W>
__device__ __forceinline__ void store_floats(T *p, const float (&f)[W])
{
    if constexpr (W == 8) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
            *(reinterpret_cast<float4 *>(p) + 1) = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            *reinterpret_cast<uint4 *>(p) = make_uint4(pack2(f[0], f[1], T()), pack2(f[2], f[3], T()), pack2(f[4], f[5], T()), pack2(f[6], f[7], T()));
        }
    } else if constexpr (W == 2) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float2 *>(p) = make_float2(f[0], f[1]);
        else *reinterpret_cast<uint32_t *>(p) = pack2(f[0], f[1], T());
    } else {
        from_float(f[0], p[0]);
    }
}
#endif

}  // namespace qnn
