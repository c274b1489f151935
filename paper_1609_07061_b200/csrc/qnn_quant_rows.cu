// Rows of real values -> int8 codes and one scale a row: plain rows, a root-mean-square norm with the residual's
// addition, a gated activation.
//
//   t[k]  = x[k]                                          (plain)
//         = s[k] gamma[k] rstd,  s = x + residual,  rstd = 1 / sqrt(mean s^2 + eps)   (norm)
//         = gate[k] / (1 + exp(-gate[k])) * up[k]         (gate)
//   scale = max|t| / 127,  code = rn(t * 127 / max|t|)
//
// In the norm rstd is one positive number of the row, so it cancels in the codes: code = rn(u * 127 / max|u|) with
// u = s gamma, and scale = rstd * max|u| / 127.  Sum of squares and maximum are then ONE reduction over the row, and a
// row that stays in registers is read once and written once.
//
// Bound by HBM: 16-bit x and residual in, 16-bit sum, 8-bit codes and their 16-bit values out is 9 bytes an element; norm
// 8192 x 4096 bf16 49 us (6.2 TB/s), gate 4096 x 12288 f16 53 us (6.6 TB/s; kept up for seconds, the power limit: 59), plain
// 8192 x 4096 fp32 25 us (6.6 TB/s), one row of 4096 2.1 us.
#include "qnn_types.cuh"

namespace qnn {
namespace {

enum RowOp { ROW_PLAIN = 0, ROW_NORM = 1, ROW_GATE = 2 };

struct RowArgs {
    const void *x;                 // x, or the gate
    const void *b;                 // residual (may be NULL), or up
    const void *gamma;             // may be NULL
    int64_t ldx, ldb;
    int64_t rows;
    int32_t K, KP;                 // KP = K rounded up to 32: codes are written up to there
    float eps;
    uint8_t *codes; int64_t ldq;
    float *scale;
    void *sum; int64_t ld_sum;     // may be NULL
    void *values; int64_t ld_values; int values_type;   // may be NULL
    int tpr;                       // threads per row, a multiple of 32
    float one;                     // 1, from memory: see to_codes
};

// 1.5 * 2^23: x + MAGIC rounds to a whole number (to even at ties) and leaves it in the low bits of the float
constexpr float MAGIC = 12582912.0f;

// two to the power, and reciprocal, on the special-function unit; results below the normal range are 0
__device__ __forceinline__ float exp2_sfu(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float rcp_sfu(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
// a / (1 + e^-a).  The reciprocal is taken of a quarter of the sum, which stays below 2^126 as long as e^-a is finite (a > -88.72):
// of the sum itself it would be 0 from a = -87.3 on, where 1e-36 is left.  Below -88.72 the sum is infinite and its reciprocal 0, as
// in the formula (but -inf gives -inf * 0, a NaN).
__device__ __forceinline__ float silu(float a) { return a * (0.25f * rcp_sfu(fmaf(0.25f, exp2_sfu(a * -1.4426950408889634f), 0.25f))); }

// what the reduction leaves a thread with: the factor that turns t into codes, the scale, and a mask for the codes
struct RowScale {
    float inv, scale;
    uint32_t keep;
};
// Below this mean square (plus eps) the fp32 sum may have lost squares to the end of the range, 2^-149; above it what is lost
// is less than 2^-52 of the sum.
constexpr float LEAST_MEAN = 1.2621774e-29f;             // 2^-96
// The sum of squares of such a row times 2^180, added up in 64 bits by every warp of the row for itself.
template <typename T>
__device__ __forceinline__ float square_sum_again(const T *x, const T *b, int32_t K)
{
    double ss = 0.0;
#pragma unroll 1
    for (int32_t k = threadIdx.x & 31; k < K; k += 32) {
        float s = to_float(x[k]);
        if (b != nullptr) s += to_float(b[k]);
        ss = fma((double)s, (double)s, ss);
    }
#pragma unroll 1
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    return (float)(ss * 0x1p180);
}
// again(): square_sum_again of the row, only called where eps is below LEAST_MEAN
template <int OP, class Again>
__device__ __forceinline__ RowScale row_scale(float ss, uint32_t top_bits, int32_t K, float eps, const Again &again)
{
    RowScale r;
    const float top = __uint_as_float(top_bits);
    r.inv = 0.0f; r.scale = 0.0f; r.keep = 0xffffffffu;
    // bits above those of the largest finite float: an infinity or a NaN
    bool bad = top_bits > 0x7f7fffffu;
    if (OP == ROW_NORM) bad = bad || !(ss <= 3.402823466e38f);
    if (bad) {
        r.scale = __uint_as_float(0x7fc00000u);
        r.keep = 0u;
    } else if (top >= 3.0092655e-36f) {      // 2^-118: below it 127 / top may overflow, and the row counts as zero
        r.inv = 127.0f / top;
        r.scale = top / 127.0f;
        if (OP == ROW_NORM) {
            const float mean = ss / (float)K + eps;
            if (mean >= LEAST_MEAN) {
                r.scale *= 1.0f / sqrtf(mean);
            } else {                                     // 2^90 times the root; whichever factor comes first stays in range
                const float root = sqrtf(again() / (float)K + eps * 0x1p90f * 0x1p90f);
                r.scale = top < 1.0f ? r.scale * 0x1p90f / root : r.scale / root * 0x1p90f;
            }
        }
    }
    return r;
}

template <int W>
__device__ __forceinline__ void store_codes(uint8_t *dst, const float (&f)[W], uint32_t keep)
{
    // f holds MAGIC + code: the code is the low byte
    if constexpr (W == 8) {
        uint32_t o[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t lo = __byte_perm(__float_as_uint(f[4 * h]), __float_as_uint(f[4 * h + 1]), 0x0040);
            const uint32_t hi = __byte_perm(__float_as_uint(f[4 * h + 2]), __float_as_uint(f[4 * h + 3]), 0x0040);
            o[h] = __byte_perm(lo, hi, 0x5410) & keep;
        }
        *reinterpret_cast<uint2 *>(dst) = make_uint2(o[0], o[1]);
    } else if constexpr (W == 2) {
        *reinterpret_cast<uint16_t *>(dst) = (uint16_t)(__byte_perm(__float_as_uint(f[0]), __float_as_uint(f[1]), 0x0040) & keep);
    } else {
        *dst = (uint8_t)(__float_as_uint(f[0]) & keep);
    }
}

template <int W>
__device__ __forceinline__ void store_values(const RowArgs &p, int64_t row, int32_t k0, const float (&f)[W])
{
    const int64_t at = row * p.ld_values + k0;
    if (p.values_type == QNN_TYPE_BF16) store_floats<__nv_bfloat16, W>(static_cast<__nv_bfloat16 *>(p.values) + at, f);
    else if (p.values_type == QNN_TYPE_F16) store_floats<__half, W>(static_cast<__half *>(p.values) + at, f);
    else store_floats<float, W>(static_cast<float *>(p.values) + at, f);
}

// t of one piece; adds to the sum of squares, and gives the sum s of the norm in `s`; weights(gv) loads the piece's gamma
template <int OP, typename T, int W, class Weights>
__device__ __forceinline__ void row_op(const RowArgs &p, const Piece<T, W> &xv, const Piece<T, W> &bv, float (&s)[W], float (&t)[W], f32x2 &ss,
                                       const Weights &weights)
{
    float x[W], b[W];
    piece_to_floats<T, W>(xv, x);
    if (OP == ROW_GATE || (OP == ROW_NORM && p.b != nullptr)) piece_to_floats<T, W>(bv, b);
    if (OP == ROW_PLAIN) {
#pragma unroll
        for (int i = 0; i < W; ++i) t[i] = x[i];
    } else if (OP == ROW_GATE) {
        if constexpr (W == 1) {
            t[0] = silu(x[0]) * b[0];
        } else {
#pragma unroll
            for (int i = 0; i < W; i += 2) {             // the same on pairs
                const f32x2 quarter = pair(0.25f, 0.25f);
                const f32x2 a2 = pair(x[i], x[i + 1]);
                float e0, e1, d0, d1;
                unpair(mul2(a2, pair(-1.4426950408889634f, -1.4426950408889634f)), e0, e1);
                unpair(fma2(quarter, pair(exp2_sfu(e0), exp2_sfu(e1)), quarter), d0, d1);
                unpair(mul2(mul2(a2, mul2(quarter, pair(rcp_sfu(d0), rcp_sfu(d1)))), pair(b[i], b[i + 1])), t[i], t[i + 1]);
            }
        }
    } else {
        float g[W];
        if (p.gamma != nullptr) {
            Piece<T, W> gv;
            weights(gv);
            piece_to_floats<T, W>(gv, g);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) g[i] = 1.0f;
        }
        if constexpr (W == 1) {
            s[0] = p.b != nullptr ? x[0] + b[0] : x[0];
            ss = fma2(pair(s[0], 0.0f), pair(s[0], 0.0f), ss);
            t[0] = s[0] * g[0];
        } else {
#pragma unroll
            for (int i = 0; i < W; i += 2) {
                f32x2 s2 = pair(x[i], x[i + 1]);
                if (p.b != nullptr) s2 = add2(s2, pair(b[i], b[i + 1]));
                unpair(s2, s[i], s[i + 1]);
                ss = fma2(s2, s2, ss);
                unpair(mul2(s2, pair(g[i], g[i + 1])), t[i], t[i + 1]);
            }
        }
    }
}
// MAGIC + code of W elements, and the values the codes stand for.  The product is rounded to fp32 before MAGIC is added, as the
// definition says; fused into one operation, t = max / 2 (63.5, common among 16-bit values) follows the rounding error of 127 / max
// to 63 or 64 instead of being a tie.  (ptxas fuses mul.rn.f32x2 and add.rn.f32x2: the sum is a fused operation of its own,
// product * one + MAGIC, with a `one` that only the host knows.)
template <int W>
__device__ __forceinline__ void to_codes(const float (&t)[W], float inv, float one, float (&f)[W])
{
    if constexpr (W == 1) {
        f[0] = __fadd_rn(__fmul_rn(t[0], inv), MAGIC);
    } else {
#pragma unroll
        for (int i = 0; i < W; i += 2) unpair(fma2(mul2(pair(t[i], t[i + 1]), pair(inv, inv)), pair(one, one), pair(MAGIC, MAGIC)), f[i], f[i + 1]);
    }
}
// the same with single sums: an instruction more for two elements, four registers less
template <int W>
__device__ __forceinline__ void to_codes_lean(const float (&t)[W], float inv, float (&f)[W])
{
    if constexpr (W == 1) {
        f[0] = __fadd_rn(__fmul_rn(t[0], inv), MAGIC);
    } else {
#pragma unroll
        for (int i = 0; i < W; i += 2) {
            unpair(mul2(pair(t[i], t[i + 1]), pair(inv, inv)), f[i], f[i + 1]);
            f[i] = __fadd_rn(f[i], MAGIC);
            f[i + 1] = __fadd_rn(f[i + 1], MAGIC);
        }
    }
}
template <int W>
__device__ __forceinline__ void to_values(float (&f)[W], float scale)
{
    if constexpr (W == 1) {
        f[0] = (f[0] - MAGIC) * scale;
    } else {
#pragma unroll
        for (int i = 0; i < W; i += 2)
            unpair(mul2(add2(pair(f[i], f[i + 1]), pair(-MAGIC, -MAGIC)), pair(scale, scale)), f[i], f[i + 1]);
    }
}
__device__ __forceinline__ float pair_sum(f32x2 v)
{
    float a, b;
    unpair(v, a, b);
    return a + b;
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// the row's sum of squares and maximum from those of its n <= 16 warps, in every lane: lane l looks at warp l's (a loop over the
// warps: gate 4096 x 12288 61.0 against 59.1 us kept up for seconds, norm 1 x 4096 2.1 against 1.9)
template <int OP>
__device__ __forceinline__ void join_warps(const float *sh_ss, const uint32_t *sh_top, int w0, int n, float &ss, uint32_t &top)
{
    const int lane = threadIdx.x & 31;
    top = __reduce_max_sync(0xffffffffu, lane < n ? sh_top[w0 + lane] : 0u);
    if (OP == ROW_NORM) {
        ss = lane < n ? sh_ss[w0 + lane] : 0.0f;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        ss = __shfl_sync(0xffffffffu, ss, 0);
    }
}

// A row of at most 8 * NV * tpr elements in registers: tpr threads own pieces of W elements, interleaved, so that a
// warp's accesses are contiguous.  W divides K; W = 8 needs 16-byte aligned rows, W = 2 aligned pairs, W = 1 nothing.
// (A kernel that also took rows ending inside a piece spent 41 instructions an element instead of 27 on the 8192 x 4096
// norm: the element-wise ends of every load and store are predicated, not branched around.)
template <int OP, typename T, int W, int NV, int MAXREG = 128>
__global__ void __launch_bounds__(512) __maxnreg__(MAXREG) row_quant_kernel(const RowArgs p)
{
    constexpr int P = NV * 8 / W;                        // pieces per thread
    constexpr int CH0 = W == 8 ? (sizeof(T) == 4 ? 2 : 4) : 8;   // pieces whose loads are in flight together
    constexpr int CH = P < CH0 ? P : CH0;
    __shared__ float sh_ss[16];
    __shared__ uint32_t sh_top[16];
    griddep_wait();

    const int tpr = p.tpr;
    const int sub = threadIdx.x / tpr, t0 = threadIdx.x - sub * tpr;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / tpr) + sub;
    const bool live = row < p.rows;
    const T *xr = static_cast<const T *>(p.x) + (live ? row : 0) * p.ldx;
    const T *br = static_cast<const T *>(p.b) + (live ? row : 0) * p.ldb;
    const bool with_b = OP == ROW_GATE || (OP == ROW_NORM && p.b != nullptr);
    const int32_t K = live ? p.K : 0;

    float t[P][W];
    f32x2 ss2 = 0ull;
    float topf = 0.0f;
#pragma unroll
    for (int c = 0; c < P; c += CH) {
        Piece<T, W> xv[CH], bv[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t k0 = ((c + j) * tpr + t0) * W;
            if (k0 < K) {
                load_piece<T, W>(xr + k0, xv[j]);
                if (with_b) load_piece<T, W>(br + k0, bv[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t k0 = ((c + j) * tpr + t0) * W;
            if (k0 < K) {
                float s[W];
                row_op<OP, T, W>(p, xv[j], bv[j], s, t[c + j], ss2,
                                 [&](Piece<T, W> &gv) { load_piece<T, W>(static_cast<const T *>(p.gamma) + k0, gv); });
                if (OP == ROW_NORM && p.sum != nullptr) store_floats<T, W>(static_cast<T *>(p.sum) + row * p.ld_sum + k0, s);
#pragma unroll
                for (int i = 0; i < W; ++i) topf = max_nan(topf, fabsf(t[c + j][i]));
            } else {
#pragma unroll
                for (int i = 0; i < W; ++i) t[c + j][i] = 0.0f;
            }
        }
    }

    // the row is in: the next kernel may be scheduled now (allowed to start at once, its blocks pile up on the free SMs)
    griddep_launch_dependents();
    float ss = 0.0f;
    if (OP == ROW_NORM) ss = warp_sum(pair_sum(ss2));
    uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(topf) & 0x7fffffffu);
    if (tpr > 32) {
        const int warp = threadIdx.x >> 5;
        if ((threadIdx.x & 31) == 0) { if (OP == ROW_NORM) sh_ss[warp] = ss; sh_top[warp] = top; }
        __syncthreads();
        join_warps<OP>(sh_ss, sh_top, sub * (tpr >> 5), tpr >> 5, ss, top);
    }
    if (!live) return;
    const RowScale r = row_scale<OP>(ss, top, p.K, p.eps, [&] { return square_sum_again<T>(xr, br, p.K); });
    if (t0 == 0) p.scale[row] = r.scale;
    uint8_t *cr = p.codes + row * p.ldq;
#pragma unroll
    for (int c = 0; c < P; ++c) {
        const int32_t k0 = (c * tpr + t0) * W;
        if (k0 < p.KP) {
            float f[W];
            to_codes<W>(t[c], r.inv, p.one, f);
            store_codes<W>(cr + k0, f, r.keep);
            if (p.values != nullptr && k0 < K) {
                to_values<W>(f, r.scale);
                store_values<W>(p, row, k0, f);
            }
        }
    }
}

// ---- rows that start or end inside 16 bytes ----------------------------------------------------------------------

// bytes sh .. sh + 15 of the 32 bytes lo, hi
template <int ES>
__device__ __forceinline__ uint4 shift_units(const uint4 &lo, const uint4 &hi, int sh)
{
    const uint32_t in[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    uint32_t a[6], b[5];
#pragma unroll
    for (int i = 0; i < 6; ++i) a[i] = sh & 8 ? in[i + 2] : in[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) b[i] = sh & 4 ? a[i + 1] : a[i];
    if (ES == 4) return make_uint4(b[0], b[1], b[2], b[3]);
    const uint32_t sel = sh & 2 ? 0x5432u : 0x3210u;
    return make_uint4(__byte_perm(b[0], b[1], sel), __byte_perm(b[1], b[2], sel), __byte_perm(b[2], b[3], sel), __byte_perm(b[3], b[4], sel));
}
// A row of a real tensor as aligned 16-byte units.
template <typename T>
struct UnitRow {
    static constexpr int E = 16 / (int)sizeof(T);
    const T *row;
    int32_t K;
    int off;                // bytes from the unit that the row starts in to its start
    bool before, after;     // the rest of its first / last unit is the tensor's too (another row, or the gap to it)
    __device__ __forceinline__ UnitRow(const void *p, int64_t r, int64_t ld, int64_t rows, int32_t k)
        : row(static_cast<const T *>(p) + r * ld), K(k), off((int)(reinterpret_cast<uintptr_t>(row) & 15u)), before(r > 0), after(r + 1 < rows) {}
    // whether all units of a warp's piece from element k on are the row's own (k: the same in all lanes)
    __device__ __forceinline__ bool inside(int32_t k) const { return (k > 0 || off == 0) && k + 256 + E <= K; }
    // the aligned 16 bytes that begin at element k; elements from K on are 0, those before the row anything
    __device__ __forceinline__ uint4 load(int32_t k) const
    {
        if (k >= 0 && k <= K - E) return *reinterpret_cast<const uint4 *>(row + k);
        if (k >= K) return make_uint4(0u, 0u, 0u, 0u);
        if ((k >= 0 || before) && (k <= K - E || after)) {
            uint4 v = *reinterpret_cast<const uint4 *>(row + k);
            const int left = (K - k) * (int)sizeof(T);
            auto keep = [&](int at) { const int n = left - at; return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u; };
            v.x &= keep(0); v.y &= keep(4); v.z &= keep(8); v.w &= keep(12);
            return v;
        }
        return load_edge(k);
    }
    // element by element: the unit reaches beyond the tensor
    __device__ __forceinline__ uint4 load_edge(int32_t k) const
    {
        uint32_t e[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            e[i] = 0u;
            if (k + i >= 0 && k + i < K) {
                if constexpr (sizeof(T) == 4) e[i] = reinterpret_cast<const uint32_t *>(row)[k + i];
                else e[i] = reinterpret_cast<const uint16_t *>(row)[k + i];
            }
        }
        if constexpr (sizeof(T) == 4) return make_uint4(e[0], e[1], e[2], e[3]);
        else return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    }
};
// 16 aligned bytes to element k on of a row; elements outside 0 .. K - 1 are not stored
template <typename T>
__device__ __forceinline__ void store_unit(T *row, int32_t k, uint4 v, int32_t K)
{
    constexpr int E = 16 / (int)sizeof(T);
    if (k >= 0 && k <= K - E) {
        *reinterpret_cast<uint4 *>(row + k) = v;
    } else if (k < K) {
        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (k + i >= 0 && k + i < K) {
                if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(row)[k + i] = x[i];
                else reinterpret_cast<uint16_t *>(row)[k + i] = (uint16_t)(i & 1 ? x[i / 2] >> 16 : x[i / 2]);
            }
        }
    }
}

// eight elements from k0 (a multiple of 8) on: the units they lie in, then shifted
template <typename T>
struct Units {
    static constexpr int N = (int)sizeof(T) / 2;         // units of a piece
    uint4 u[N + 1];
    __device__ __forceinline__ void load(const UnitRow<T> &r, int32_t k0, bool inside)
    {
        const int32_t k = k0 - r.off / (int)sizeof(T);
        if (inside) {                                    // (all lanes)
            const uint4 *at = reinterpret_cast<const uint4 *>(r.row + k);
#pragma unroll
            for (int n = 0; n <= N; ++n) u[n] = at[n];
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) u[n] = r.load(k + n * r.E);
            u[N] = r.off != 0 ? r.load(k + 8) : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    __device__ __forceinline__ void piece(int off, Piece<T, 8> &v) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint4 x = shift_units<(int)sizeof(T)>(u[n], u[n + 1], off);
            v.w[4 * n] = x.x; v.w[4 * n + 1] = x.y; v.w[4 * n + 2] = x.z; v.w[4 * n + 3] = x.w;
        }
    }
};
// Stores a warp's pieces of a row, piece by piece along it, lanes side by side: a unit of memory is put together from a lane's
// elements and those of the lane before, so that all but a row's ends are whole aligned stores.
template <typename T>
struct RunStore {
    static constexpr int N = (int)sizeof(T) / 2, E = 16 / (int)sizeof(T);
    T *row;
    int off;
    int32_t K;
    uint4 last;             // the last unit of this lane's piece before (of lane 31 at first: of the warp before)
    uint4 held;             // lane 0: its first unit, when the one before it is not known yet
    __device__ __forceinline__ RunStore(T *r, int32_t k)
        : row(r), off((int)(reinterpret_cast<uintptr_t>(r) & 15u)), K(k), last(make_uint4(0u, 0u, 0u, 0u)), held(last) {}
    static __device__ __forceinline__ void pack(const float (&f)[8], uint4 (&u)[N])
    {
        if constexpr (N == 1) {
            u[0] = make_uint4(pack2(f[0], f[1], T()), pack2(f[2], f[3], T()), pack2(f[4], f[5], T()), pack2(f[6], f[7], T()));
        } else {
            u[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            u[N - 1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
        }
    }
    // hold: keep the run's first unit for release()
    __device__ __forceinline__ void put(const float (&f)[8], int32_t k0, bool hold)
    {
        const int lane = threadIdx.x & 31;
        const bool inside = (k0 - lane * 8 > 0 || off == 0) && k0 - lane * 8 + 256 <= K;
        uint4 u[N];
        pack(f, u);
        if (off == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (inside) *reinterpret_cast<uint4 *>(row + k0 + n * E) = u[n];
                else store_unit<T>(row, k0 + n * E, u[n], K);
            }
            return;
        }
        const int from = (lane + 31) & 31;
        const bool top = lane == 31;
        uint4 before;
        before.x = __shfl_sync(0xffffffffu, top ? last.x : u[N - 1].x, from);
        before.y = __shfl_sync(0xffffffffu, top ? last.y : u[N - 1].y, from);
        before.z = __shfl_sync(0xffffffffu, top ? last.z : u[N - 1].z, from);
        before.w = __shfl_sync(0xffffffffu, top ? last.w : u[N - 1].w, from);
        last = u[N - 1];
        if (hold) held = u[0];
        const int32_t k = k0 - off / (int)sizeof(T);
        const uint4 x = shift_units<(int)sizeof(T)>(before, u[0], 16 - off), y = shift_units<(int)sizeof(T)>(u[0], u[N - 1], 16 - off);
        if (inside) {
            if (!(hold && lane == 0)) *reinterpret_cast<uint4 *>(row + k) = x;
            if (N == 2) *reinterpret_cast<uint4 *>(row + k + E) = y;
        } else {
            if (!(hold && lane == 0)) store_unit<T>(row, k, x, K);
            if (N == 2) store_unit<T>(row, k + E, y, K);
        }
        // the row ends here: what lies past the last unit
        if (top && k0 + 8 >= K && k + 8 < K)
            store_unit<T>(row, k + 8, shift_units<(int)sizeof(T)>(u[N - 1], make_uint4(0u, 0u, 0u, 0u), 16 - off), K);
    }
    __device__ __forceinline__ void release(int32_t first, const uint4 &before)
    {
        if ((threadIdx.x & 31) == 0 && off != 0)
            store_unit<T>(row, first - off / (int)sizeof(T), shift_units<(int)sizeof(T)>(before, held, 16 - off), K);
    }
};

// A row of any alignment in registers: a warp owns a run of P * 256 elements, lane by lane eight, and the real tensors move in
// aligned units of 16 bytes whatever their offsets, which may differ from tensor to tensor.  A unit's elements are shifted
// into place by selects and byte permutes (15 a unit and direction, 37 instructions an element where whole vectors take 23).  Half
// the issue slots are used and loads are the first thing waited for: registers hold what is in flight, and their number lets two
// blocks of 350 threads run on an SM (gate 3000 x 11009 116 us without the limits).  3000 x 11009 bf16: norm 112 us (2.7 TB/s), gate
// 71 us (3.3 TB/s); element by element 148 and 119.
template <int OP, typename T, int P, int MAXREG = P == 4 ? 80 : 64>
__global__ void __launch_bounds__(512) __maxnreg__(MAXREG) row_quant_ragged_kernel(const RowArgs p)
{
    constexpr int CH = P == 1 || sizeof(T) == 4 ? 1 : 2; // pieces whose loads are in flight together
    __shared__ float sh_ss[16];
    __shared__ uint32_t sh_top[16];
    // what the next warp needs to complete the first units of its run: t of a run's last eight elements, their last unit of sums
    __shared__ float4 sh_t[16][2];
    __shared__ uint4 sh_sum[16];
    griddep_wait();

    const int tpr = p.tpr, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = threadIdx.x / tpr, w = (threadIdx.x - sub * tpr) >> 5;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / tpr) + sub;
    const bool live = row < p.rows;
    const int64_t rr = live ? row : 0;
    const int32_t K = live ? p.K : 0, first = w * (P * 256);
    const bool with_b = OP == ROW_GATE || (OP == ROW_NORM && p.b != nullptr);
    const UnitRow<T> xr(p.x, rr, p.ldx, p.rows, K), br(p.b, rr, p.ldb, p.rows, K), gr(p.gamma, 0, 0, 1, K);

    float t[P][8];
    f32x2 ss2 = 0ull;
    float topf = 0.0f;
    const bool keep_sum = OP == ROW_NORM && p.sum != nullptr;
    RunStore<T> sums(static_cast<T *>(p.sum) + (keep_sum ? rr : 0) * p.ld_sum, K);
#pragma unroll
    for (int c = 0; c < P; c += CH) {
        Units<T> xv[CH], bv[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t k = first + (c + j) * 256;
            if (k < K) {
                xv[j].load(xr, k + lane * 8, xr.inside(k));
                if (with_b) bv[j].load(br, k + lane * 8, br.inside(k));
            }
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t k = first + (c + j) * 256;
            if (k < K) {                                 // (elements from K on are zeros, and give t = 0)
                float s[8];
                Piece<T, 8> xp, bp;
                xv[j].piece(xr.off, xp);
                if (with_b) bv[j].piece(br.off, bp);
                row_op<OP, T, 8>(p, xp, bp, s, t[c + j], ss2, [&](Piece<T, 8> &gv) {
                    Units<T> g;
                    g.load(gr, k + lane * 8, gr.inside(k));
                    g.piece(gr.off, gv);
                });
                if (keep_sum) sums.put(s, k + lane * 8, c + j == 0 && w > 0);
#pragma unroll
                for (int i = 0; i < 8; ++i) topf = max_nan(topf, fabsf(t[c + j][i]));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) t[c + j][i] = 0.0f;
            }
        }
    }

    griddep_launch_dependents();
    float ss = 0.0f;
    if (OP == ROW_NORM) ss = warp_sum(pair_sum(ss2));
    uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(topf) & 0x7fffffffu);
    if (tpr > 32) {
        if (lane == 0) { if (OP == ROW_NORM) sh_ss[warp] = ss; sh_top[warp] = top; }
        if (lane == 31) {
            sh_t[warp][0] = make_float4(t[P - 1][0], t[P - 1][1], t[P - 1][2], t[P - 1][3]);
            sh_t[warp][1] = make_float4(t[P - 1][4], t[P - 1][5], t[P - 1][6], t[P - 1][7]);
            if (keep_sum) sh_sum[warp] = sums.last;
        }
        __syncthreads();
        join_warps<OP>(sh_ss, sh_top, sub * (tpr >> 5), tpr >> 5, ss, top);
        if (keep_sum && w > 0 && first < K) sums.release(first, sh_sum[warp - 1]);
    }
    if (!live) return;
    const RowScale r = row_scale<OP>(ss, top, p.K, p.eps, [&] { return square_sum_again<T>(xr.row, br.row, p.K); });
    if (w == 0 && lane == 0) p.scale[row] = r.scale;
    uint8_t *cr = p.codes + row * p.ldq;
    auto finish = [&](auto type) {
        using V = decltype(type);
        RunStore<V> values(static_cast<V *>(p.values) + (p.values != nullptr ? row * p.ld_values : 0), K);
        if (p.values != nullptr && w > 0 && values.off != 0) {
            const float4 a = sh_t[warp - 1][0], b = sh_t[warp - 1][1];
            const float e[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            float f[8];
            uint4 u[RunStore<V>::N];
            to_codes<8>(e, r.inv, p.one, f);
            to_values<8>(f, r.scale);
            RunStore<V>::pack(f, u);
            values.last = u[RunStore<V>::N - 1];
        }
#pragma unroll
        for (int c = 0; c < P; ++c) {
            const int32_t k = first + c * 256, k0 = k + lane * 8;
            if (k >= p.KP) break;
            float f[8];
            to_codes<8>(t[c], r.inv, p.one, f);
            if (k0 < p.KP) store_codes<8>(cr + k0, f, r.keep);
            if (p.values != nullptr && k < K) {
                to_values<8>(f, r.scale);
                values.put(f, k0, false);
            }
        }
    };
    if (p.values_type == QNN_TYPE_BF16) finish(__nv_bfloat16());
    else if (p.values_type == QNN_TYPE_F16) finish(__half());
    else finish(float());
}

// Rows longer than the registers of a block hold: two passes over the row, the second mostly from L2.  sum_out may be x
// or residual, so the first pass writes nothing and the second writes each element after reading it.
// AGAIN: rows of a norm may need their sum of squares a second time (left to where eps allows it: the path costs registers).
// What is read comes from blocks that share an SM; where the compiler would take the registers of one of them, it is held to as
// many blocks as fit otherwise (2000 rows: norm 33000 bf16 122 us with two blocks, 172 with one; norm 11010 fp32 79.5 / 88; gate
// 33000 fp32 150 / 179; plain 33000 bf16 46 / 54).
template <typename T, int W>
constexpr int long_blocks(int op)
{
    if (W == 8 && op == (sizeof(T) == 4 ? ROW_GATE : ROW_NORM)) return 2;
    if (op == ROW_NORM ? W == 2 && sizeof(T) == 4 : op == ROW_PLAIN && W == 8 && sizeof(T) == 2) return 3;
    return 0;                                            // (no such demand)
}
template <int OP, typename T, int W, bool AGAIN>
__global__ void __launch_bounds__(512, (long_blocks<T, W>(OP))) row_quant_long_kernel(const RowArgs p)
{
    __shared__ float sh_ss[16];
    __shared__ uint32_t sh_top[16];
    griddep_wait();
    const int64_t row = blockIdx.x;
    const T *xr = static_cast<const T *>(p.x) + row * p.ldx;
    const T *br = static_cast<const T *>(p.b) + row * p.ldb;
    const bool with_b = OP == ROW_GATE || (OP == ROW_NORM && p.b != nullptr);
    const int64_t step = (int64_t)blockDim.x * W;
    f32x2 ss2 = 0ull;
    float topf = 0.0f;
    // CH pieces a round, their loads in flight together (narrow ones: gate 2000 x 28002 bf16 in pairs 113 us with four, 153 with two;
    // the norm, with gamma's besides, 78 and 70)
    constexpr int CH = W < 8 && OP != ROW_NORM ? 4 : 2;
    for (int64_t k = (int64_t)threadIdx.x * W; k < p.K; k += CH * step) {
        Piece<T, W> xv[CH], bv[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t k0 = k + c * step;
            if (k0 < p.K) {
                load_piece<T, W>(xr + k0, xv[c]);
                if (with_b) load_piece<T, W>(br + k0, bv[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t k0 = k + c * step;
            if (k0 < p.K) {
                float s[W], t[W];
                row_op<OP, T, W>(p, xv[c], bv[c], s, t, ss2,
                                 [&](Piece<T, W> &gv) { load_piece<T, W>(static_cast<const T *>(p.gamma) + k0, gv); });
#pragma unroll
                for (int i = 0; i < W; ++i) topf = max_nan(topf, fabsf(t[i]));
            }
        }
    }
    float ss = 0.0f;
    if (OP == ROW_NORM) ss = warp_sum(pair_sum(ss2));
    uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(topf) & 0x7fffffffu);
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) { if (OP == ROW_NORM) sh_ss[warp] = ss; sh_top[warp] = top; }
    __syncthreads();
    griddep_launch_dependents();
    join_warps<OP>(sh_ss, sh_top, 0, (int)(blockDim.x >> 5), ss, top);
    const RowScale r = row_scale<OP>(ss, top, p.K, p.eps, [&] {
        float again = ss;
        if constexpr (AGAIN) {
            again = square_sum_again<T>(xr, br, p.K);
            __syncthreads();                             // (the block is one row) nobody writes the sums over x before all have read it
        }
        return again;
    });
    if (threadIdx.x == 0) p.scale[row] = r.scale;
    uint8_t *cr = p.codes + row * p.ldq;
    for (int64_t k = (int64_t)threadIdx.x * W; k < p.KP; k += CH * step) {
        Piece<T, W> xv[CH], bv[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t k0 = k + c * step;
            if (k0 < p.K) {
                load_piece<T, W>(xr + k0, xv[c]);
                if (with_b) load_piece<T, W>(br + k0, bv[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t k0 = k + c * step;
            if (k0 >= p.KP) break;
            float s[W], t[W], f[W];
            f32x2 unused = 0ull;
#pragma unroll
            for (int i = 0; i < W; ++i) t[i] = 0.0f;
            if (k0 < p.K) {
                row_op<OP, T, W>(p, xv[c], bv[c], s, t, unused,
                                 [&](Piece<T, W> &gv) { load_piece<T, W>(static_cast<const T *>(p.gamma) + k0, gv); });
                if (OP == ROW_NORM && p.sum != nullptr) store_floats<T, W>(static_cast<T *>(p.sum) + row * p.ld_sum + k0, s);
            }
            if constexpr (OP == ROW_GATE) to_codes<W>(t, r.inv, p.one, f);   // (gate 2000 x 28002 bf16 113 us, lean 132; plain 33002 114, 89)
            else to_codes_lean<W>(t, r.inv, f);
            store_codes<W>(cr + k0, f, r.keep);
            if (p.values != nullptr && k0 < p.K) {
                to_values<W>(f, r.scale);
                store_values<W>(p, row, (int32_t)k0, f);
            }
        }
    }
}

constexpr int MAX_TPR = 512;

template <int OP, typename T, int W>
int launch_rows(RowArgs p, const char *what, cudaStream_t st, bool two_passes = false)
{
    // (narrow accesses: more instructions an element, so long rows take the rolled loops of the other kernel)
    constexpr int MAX_NV = W == 8 ? 8 : 2;
    constexpr int64_t MAX_GROUPS = W == 8 ? (int64_t)MAX_TPR * MAX_NV : W == 2 ? 1024 : 256;
    const int64_t groups = ceil_div(p.KP, 8);            // a row in units of eight elements
    if (groups > MAX_GROUPS || two_passes) {
        if constexpr (OP == ROW_NORM) {
            if (p.eps < LEAST_MEAN) {
                QNN_CUDA(launch_pdl(row_quant_long_kernel<OP, T, W, true>, dim3((unsigned)p.rows), dim3(512), 0, st, p));
                return check_launch(what);
            }
        }
        QNN_CUDA(launch_pdl(row_quant_long_kernel<OP, T, W, false>, dim3((unsigned)p.rows), dim3(512), 0, st, p));
        return check_launch(what);
    }
    // Groups a thread.  Few rows: one, for latency.  Many rows: two while that gives blocks of at most 128 threads; small blocks
    // stream best, so four for longer rows (norm, bf16, 8192 rows: K = 4096 48.7 against 50.9 us with two, K = 8192 92.3 against
    // 107.6; 1200 rows of 4096 11.5 against 10.6, so there two), but not in fp32, whose loads need twice the registers
    // (8192 x 4096: 80.7 against 76.3).
    const int64_t sms = sm_count();
    int nv = p.rows <= 2 * sms ? 1 : 2;
    if (nv == 2 && W == 8 && sizeof(T) == 2 && (groups > 512 || (groups > 256 && p.rows >= 16 * sms))) nv = 4;
    while (groups > (int64_t)MAX_TPR * nv) nv *= 2;
    p.tpr = (int)(ceil_div(ceil_div(groups, nv), 32) * 32);
    const int rpb = p.tpr >= 128 ? 1 : 128 / p.tpr;      // rows of short vectors share a block
    const dim3 grid((unsigned)ceil_div(p.rows, rpb)), block((unsigned)(p.tpr * rpb));
    switch (nv) {
        case 1: QNN_CUDA(launch_pdl(row_quant_kernel<OP, T, W, 1>, grid, block, 0, st, p)); break;
        case 2: QNN_CUDA(launch_pdl(row_quant_kernel<OP, T, W, 2>, grid, block, 0, st, p)); break;
        case 4:
            if constexpr (OP == ROW_GATE && W == 8 && sizeof(T) == 2) {
                // 64 registers a thread let 1024 threads of an SM run: two blocks of 352 or 384 (K of 10241 to 12288), a quarter or
                // more of them idle.  56 let three run, at the price of a few spills (4096 x 12288 f16: 52.9 against 58.8 us, 4096 x
                // 10496 bf16 49 against 56).  Other blocks fill at least 820 of the 1024.
                if (1024 / block.x * block.x < 820) {
                    QNN_CUDA(launch_pdl(row_quant_kernel<OP, T, W, 4, 56>, grid, block, 0, st, p));
                    break;
                }
            }
            if constexpr (W == 8) QNN_CUDA(launch_pdl(row_quant_kernel<OP, T, W, 4>, grid, block, 0, st, p));
            break;
        default:
            if constexpr (W == 8) QNN_CUDA(launch_pdl(row_quant_kernel<OP, T, W, 8>, grid, block, 0, st, p));
            break;
    }
    return check_launch(what);
}

template <int OP, typename T>
int launch_ragged(RowArgs p, const char *what, cudaStream_t st)
{
    // Pieces a lane: one for few rows, for latency, and in fp32 (norm 4000 x 2003: 34.6 us against 40.2 with two); two else (norm
    // 4000 x 2003 bf16: 27.3 against 32.9 with one and 32.3 with four).
    const int64_t groups = ceil_div(p.KP, 8);
    int pieces = p.rows <= 2 * (int64_t)sm_count() || sizeof(T) == 4 || groups <= 32 ? 1 : 2;
    while (groups > (int64_t)MAX_TPR * pieces) pieces *= 2;
    p.tpr = (int)(ceil_div(groups, 32 * pieces) * 32);
    const int rpb = p.tpr >= 128 ? 1 : 128 / p.tpr;
    const dim3 grid((unsigned)ceil_div(p.rows, rpb)), block((unsigned)(p.tpr * rpb));
    switch (pieces) {
        case 1: QNN_CUDA(launch_pdl(row_quant_ragged_kernel<OP, T, 1>, grid, block, 0, st, p)); break;
        case 2: QNN_CUDA(launch_pdl(row_quant_ragged_kernel<OP, T, 2>, grid, block, 0, st, p)); break;
        default: QNN_CUDA(launch_pdl(row_quant_ragged_kernel<OP, T, 4>, grid, block, 0, st, p)); break;
    }
    return check_launch(what);
}

template <int OP, typename T>
int launch_rows_w(const RowArgs &p, const char *what, cudaStream_t st)
{
    // widest access that every row of every real tensor allows and that the row length is a multiple of
    auto fits = [&](size_t elems) {
        if (p.K % (int)elems != 0) return false;
        auto ok = [&](const void *q, int64_t ld, size_t es) { return q == nullptr || (aligned(q, elems * es < 16 ? elems * es : 16) && (size_t)ld % (elems * es < 16 ? elems : 16 / es) == 0); };
        const size_t vs = p.values_type == QNN_TYPE_F32 ? 4 : 2;
        return ok(p.x, p.ldx, sizeof(T)) && ok(p.b, p.ldb, sizeof(T)) && ok(p.gamma, 0, sizeof(T)) && ok(p.sum, p.ld_sum, sizeof(T)) &&
               ok(p.values, p.ld_values, vs);
    };
    if constexpr (OP == ROW_NORM) {
        // Without an eps worth the name a row may have to be read once more, and is gone by then if the sums overwrite it as they
        // are computed: the two passes write them last.  (8192 x 4096 bf16 in place with eps 0: 88 us; not in place 50.)
        if (p.eps < LEAST_MEAN && p.sum != nullptr && (p.sum == p.x || p.sum == p.b))
            return fits(8) ? launch_rows<OP, T, 8>(p, what, st, true) : fits(2) ? launch_rows<OP, T, 2>(p, what, st, true)
                                                                               : launch_rows<OP, T, 1>(p, what, st, true);
    }
    if (fits(8)) return launch_rows<OP, T, 8>(p, what, st);
    // Rows that end inside 16 bytes: in pairs where all tensors lie alike and a block's registers hold the row (bf16 norm 5000 x
    // 4098 51 us, shifted units 68; gate 39 and 49), and for the norm of many longer rows in pairs too, in two passes (2000 x
    // 11010 70 and 74); else shifted units (2000 x 11010 gate 47.5 us, 51.5 in pairs; 64 x 11010 norm 8.1, 10; 5000 x 4097 norm 70,
    // by single elements 97, gate 50, 84; 1 x 4097 norm 3.7, 6.0).  Single elements are left to the shortest rows and those that
    // no block holds (gate 2000 x 28001 200 us, in pairs 2000 x 28002 116).
    const bool pairs = fits(2), held = p.KP <= 8 * 4 * MAX_TPR;
    if (pairs && (p.KP <= 8192 || !held || (OP == ROW_NORM && p.rows > 2 * (int64_t)sm_count()))) return launch_rows<OP, T, 2>(p, what, st);
    if (held && p.KP >= 256) return launch_ragged<OP, T>(p, what, st);
    return launch_rows<OP, T, 1>(p, what, st);
}

template <int OP>
int quant_rows(RowArgs p, int type, int64_t K, const char *what, void *stream)
{
    QNN_REQUIRE(type_ok(type), QNN_ERR_INVALID_ARG, "%s: unknown element type %d", what, type);
    QNN_REQUIRE(p.rows >= 0 && K >= 0, QNN_ERR_INVALID_ARG, "%s: negative size", what);
    if (p.rows == 0) return QNN_OK;
    QNN_REQUIRE(p.rows < ((int64_t)1 << 31) && K < ((int64_t)1 << 31) - 32, QNN_ERR_UNSUPPORTED, "%s: rows or K of 2^31 and more", what);
    if (K == 0) {                                        // rows of nothing: no codes, and the scale of a row of zeros
        QNN_REQUIRE(p.scale && aligned(p.scale, 4), QNN_ERR_INVALID_ARG, "%s: scale is NULL or not aligned to its elements", what);
        QNN_CUDA(cudaMemsetAsync(p.scale, 0, (size_t)p.rows * 4, as_stream(stream)));
        return QNN_OK;
    }
    QNN_REQUIRE(p.x && p.codes && p.scale && (OP != ROW_GATE || p.b), QNN_ERR_INVALID_ARG, "%s: NULL pointer", what);
    const int64_t kp = (int64_t)round_up((size_t)K, 32);
    QNN_REQUIRE(p.ldx >= K && (!p.b || p.ldb >= K) && (!p.sum || p.ld_sum >= K), QNN_ERR_INVALID_ARG, "%s: leading dimension below K", what);
    QNN_REQUIRE(p.ldq >= kp, QNN_ERR_INVALID_ARG, "%s: ldq below K rounded up to 32", what);
    QNN_REQUIRE(aligned(p.codes, 16) && p.ldq % 16 == 0, QNN_ERR_ALIGNMENT, "%s: codes must be 16-byte aligned, ldq a multiple of 16", what);
    const size_t es = (size_t)type_bytes(type);
    QNN_REQUIRE(aligned(p.x, es) && aligned(p.b, es) && aligned(p.gamma, es) && aligned(p.sum, es) && aligned(p.scale, 4), QNN_ERR_ALIGNMENT,
                "%s: a pointer is not aligned to its elements", what);
    if (p.values) {
        QNN_REQUIRE(type_ok(p.values_type), QNN_ERR_INVALID_ARG, "%s: unknown type %d of the values", what, p.values_type);
        QNN_REQUIRE(p.ld_values >= K, QNN_ERR_INVALID_ARG, "%s: ld_values below K", what);
        QNN_REQUIRE(aligned(p.values, (size_t)type_bytes(p.values_type)), QNN_ERR_ALIGNMENT, "%s: values are not aligned to their elements", what);
    }
    if (OP == ROW_NORM) {
        QNN_REQUIRE(p.eps >= 0.0f, QNN_ERR_INVALID_ARG, "%s: eps is negative or NaN", what);
        QNN_REQUIRE(p.sum == nullptr || p.sum != p.x || p.ld_sum == p.ldx, QNN_ERR_INVALID_ARG, "%s: sum_out over x needs the same leading dimension", what);
        QNN_REQUIRE(p.sum == nullptr || p.sum != p.b || p.ld_sum == p.ldb, QNN_ERR_INVALID_ARG,
                    "%s: sum_out over the residual needs the same leading dimension", what);
    }
    p.K = (int32_t)K;
    p.KP = (int32_t)kp;
    p.one = 1.0f;
    cudaStream_t st = as_stream(stream);
    switch (type) {
        case QNN_TYPE_F32: return launch_rows_w<OP, float>(p, what, st);
        case QNN_TYPE_BF16: return launch_rows_w<OP, __nv_bfloat16>(p, what, st);
        default: return launch_rows_w<OP, __half>(p, what, st);
    }
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" {

int qnn_quantize_rows_i8(const void *x, int type, int64_t rows, int64_t K, int64_t ldx, void *codes, int64_t ldq, float *scale, void *values,
                         int values_type, int64_t ld_values, void *stream)
{
    RowArgs p{};
    p.x = x; p.ldx = ldx; p.rows = rows;
    p.codes = static_cast<uint8_t *>(codes); p.ldq = ldq; p.scale = scale;
    p.values = values; p.values_type = values_type; p.ld_values = ld_values;
    return quant_rows<ROW_PLAIN>(p, type, K, "qnn_quantize_rows_i8", stream);
}

int qnn_rmsnorm_quant_i8(const void *x, const void *residual, int type, int64_t rows, int64_t K, int64_t ldx, int64_t ldr, const void *gamma,
                         float eps, void *codes, int64_t ldq, float *scale, void *sum_out, int64_t ld_sum, void *values, int values_type,
                         int64_t ld_values, void *stream)
{
    RowArgs p{};
    p.x = x; p.ldx = ldx; p.rows = rows;
    p.b = residual; p.ldb = residual ? ldr : 0;
    p.gamma = gamma; p.eps = eps;
    p.codes = static_cast<uint8_t *>(codes); p.ldq = ldq; p.scale = scale;
    p.sum = sum_out; p.ld_sum = ld_sum;
    p.values = values; p.values_type = values_type; p.ld_values = ld_values;
    return quant_rows<ROW_NORM>(p, type, K, "qnn_rmsnorm_quant_i8", stream);
}

int qnn_silu_mul_quant_i8(const void *gate, const void *up, int type, int64_t rows, int64_t K, int64_t ldg, int64_t ldu, void *codes, int64_t ldq,
                          float *scale, void *values, int values_type, int64_t ld_values, void *stream)
{
    RowArgs p{};
    p.x = gate; p.ldx = ldg; p.rows = rows;
    p.b = up; p.ldb = ldu;
    p.codes = static_cast<uint8_t *>(codes); p.ldq = ldq; p.scale = scale;
    p.values = values; p.values_type = values_type; p.ld_values = ld_values;
    return quant_rows<ROW_GATE>(p, type, K, "qnn_silu_mul_quant_i8", stream);
}

}  // extern "C"
