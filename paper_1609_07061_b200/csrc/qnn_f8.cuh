// What the products and the weight gradient of 8-bit floating-point codes share on the host.
#pragma once
#include <atomic>
#include "qnn_types.cuh"

namespace qnn {

constexpr int MAX_GROUPS = QNN_F8_MAX_GROUPS;

// Weight gradient (qnn_gemm_f8_wgrad.cu): dw[g][n,k] from codes dy [.., N] and x [.., K] of M rows in groups.
struct WgParams {
    const uint8_t *dy, *x, *dy_scale, *x_scale;
    int64_t ld_dy, ldx, ld_dys, ld_xs, M, ld_dw;
    const int64_t *offsets;          // [groups + 1] or NULL: one group of all rows
    void *dw;
    int32_t N, K, groups, tiles_n, tiles_k;
};
int run_f8_wgrad(const char *what, WgParams p, int dy_type, int x_type, int out_type, cudaStream_t st);

namespace {

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

}  // namespace
}  // namespace qnn
