// Products of 8-bit floating-point codes: the entry points, the choice of a configuration, and the forward products' kernels (see
// qnn_gemm_f8.cuh).
#include "qnn_gemm_f8.cuh"

namespace qnn {
namespace {

// Clusters of a kernel that are resident at once, asked once per device (0: none can be launched).  Fewer than the SMs would hold: the
// GPU's groups of SMs leave some over (of eights, one CTA an SM, 15 fit).
template <int NT, int CTAS, int SPLIT>
int clusters_resident()
{
    static std::atomic<int> cached[64];                 // 0 = not asked yet; stored as clusters + 1
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int v = cached[dev].load(std::memory_order_acquire);
    if (v == 0) {
        using S = F8Cfg<NT, FORWARD, CTAS, __nv_bfloat16, SPLIT>;
        auto kern = gemm_f8_kernel<NT, FORWARD, CTAS, __nv_bfloat16, SPLIT>;
        int n = 0;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::TOTAL) == cudaSuccess) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(CTAS * SPLIT * S::RESIDENT * (unsigned)sm_count());
            cfg.blockDim = dim3(F8_THREADS);
            cfg.dynamicSmemBytes = S::TOTAL;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = CTAS * SPLIT; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr; cfg.numAttrs = 1;
            if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) { (void)cudaGetLastError(); n = 0; }
        } else {
            (void)cudaGetLastError();
        }
        v = n + 1;
        cached[dev].store(v, std::memory_order_release);
    }
    return v - 1;
}
int parts_resident(int width, int split)
{
    switch (split) {
        case 2: return width == 16 ? clusters_resident<16, 1, 2>() : clusters_resident<128, 1, 2>();
        case 4: return width == 16 ? clusters_resident<16, 1, 4>() : clusters_resident<128, 1, 4>();
        default: return width == 16 ? clusters_resident<16, 1, 8>() : clusters_resident<128, 1, 8>();
    }
}

}  // namespace

int pairs_resident_f8() { return clusters_resident<256, 2, 1>(); }

namespace {

// len: tokens of a group; groups: how many are taken to have any; rows: the tiles' other dimension; nkb: blocks of the reduction; cut: it
// may be cut.  Clocks of a launch, fitted to measured ones: a block of a tile costs what its loads do (2.2 clk for each of the 128 + n / ctas
// rows of 128 bytes that a CTA loads), or its products (2 n, at least 400); the results of a tile cost 11 clk a column, under the
// products of the next one; joining parts of a reduction costs 2500, by sends 1000.  Against every other configuration at 56 sizes: 1.5 %
// slower than the best on average, at worst 1.34 times (1254 x 3968 x 128, one block: 16.4 us, 12.3 with tiles of 128 columns).
F8Choice cheapest(int64_t len, int64_t groups, int64_t rows, int64_t nkb, bool cut)
{
    static const int widths[] = {16, 32, 64, 128, 256};
    F8Choice best = {0, 1, 1, 0};
    double cost = 0.0;
    for (int w : widths) {
        const int ctas = w == 256 ? 2 : 1, step = chunk_step(w);
        const int64_t workers = ctas == 1 ? sm_count() : pairs_resident_f8();
        if (workers < 1) continue;
        const int64_t across = ceil_div(rows, (int64_t)BM * ctas) * groups, least = ceil_div(len, w);
        for (int64_t k = least; k <= least + 3 && (k == least || ceil_div(len, k) >= step); ++k) {
            const int64_t n = (int64_t)round_up((size_t)ceil_div(len, k), (size_t)step), tiles = k * across;
            const double load = 2.2 * (128.0 + (double)n / ctas), issue = 2.0 * (double)n > 400.0 ? 2.0 * (double)n : 400.0, block = load > issue ? load : issue, drain = 11.0 * (double)n;
            for (int split = w == 16 ? 2 : 1; split <= (ctas == 1 && cut ? 8 : 1); split *= 2) {
                if (split > 1 && (nkb < 4 * split || tiles > parts_resident(w, split))) break;
                const double part = (double)ceil_div(nkb, split) * block;
                const double t = (double)ceil_div(tiles * split, workers) * (part > drain ? part : drain) + drain + (split == 1 ? 0.0 : w == 16 ? 1000.0 : 2500.0) + (ctas == 2 ? 1500.0 : 0.0);
                if (best.width == 0 || t < cost) { best = {w, ctas, split, (int)n}; cost = t; }
            }
        }
    }
    return best;
}

}  // namespace

F8Choice choose_f8(int64_t M, int64_t groups, int64_t N, int64_t nkb, bool one_group)
{
    const int64_t taken = groups < M ? groups : M;
    F8Choice k = cheapest(ceil_div(M, taken), taken, N, nkb, one_group);
    if (!one_group) k.nt = k.width;                // (groups differ: their chunks are evened out one by one)
    if (k.split > 1 && k.width == 32) k.width = 64;    // (32 columns, in the kernel for 64)
    return k;
}

namespace {

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
    return across ? run_f8_across(c, p, out_type, as_stream(stream)) : run_f8_forward(c, p, out_type, as_stream(stream));
}

}  // namespace

int run_f8_forward(const F8Call &c, const F8Params &p, int out_type, cudaStream_t st) { return run_f8<FORWARD>(c, p, out_type, st); }
int f8_forward_status(int *code)
{
    QNN_CUDA(status_read_clear(code));
    return QNN_OK;
}

int gemm_f8_status(int *code)
{
    int c[2] = {0, 0};
    if (int rc = f8_forward_status(&c[0])) return rc;
    if (int rc = f8_across_status(&c[1])) return rc;
    *code = c[0] ? c[0] : c[1];
    return QNN_OK;
}

}  // namespace qnn

using namespace qnn;

extern "C" {

int qnn_gemm_f8_kernel(int64_t M, int64_t N, int64_t K, int64_t groups)
{
    const int64_t most = (int64_t)1 << 30;
    if (M <= 0 || N <= 0 || K < 0 || groups < 0 || M > most || N > most || K > most || groups > MAX_GROUPS) return 0;
    const F8Choice k = choose_f8(M, groups ? groups : 1, N, ceil_div(K, 128), groups == 0);
    return k.width | k.split << 12 | k.nt << 16;
}

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
    WgParams p{};
    p.dy = static_cast<const uint8_t *>(dy); p.ld_dy = ld_dy; p.dy_scale = static_cast<const uint8_t *>(dy_scale); p.ld_dys = ld_dys;
    p.x = static_cast<const uint8_t *>(x); p.ldx = ldx; p.x_scale = static_cast<const uint8_t *>(x_scale); p.ld_xs = ld_xs;
    p.offsets = offsets; p.groups = (int32_t)groups;
    p.M = M; p.N = (int32_t)N; p.K = (int32_t)K;
    p.dw = dw; p.ld_dw = ld_dw;
    return run_f8_wgrad(what, p, dy_type, x_type, dw_type, as_stream(stream));
}

}  // extern "C"
