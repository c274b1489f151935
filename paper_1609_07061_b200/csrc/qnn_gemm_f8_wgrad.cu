// Products of 8-bit floating-point codes: the kernels of weight gradients (see qnn_gemm_f8.cuh).
#include "qnn_gemm_f8.cuh"

namespace qnn {

int run_f8_wgrad(const F8Call &c, const F8Params &p, int out_type, cudaStream_t st) { return run_f8<WGRAD>(c, p, out_type, st); }
int f8_wgrad_status(int *code)
{
    QNN_CUDA(status_read_clear(code));
    return QNN_OK;
}

}  // namespace qnn
