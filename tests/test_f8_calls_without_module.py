"""The 8-bit floating-point calls where the CPython module of the per-token calls cannot be built: the same refusals through ctypes."""
import pytest

from test_calls_without_module import run_without


def test_refusals_without_the_module():
    run_without("tests/test_f8_refusals.py", "tests/test_f8_calls_without_module.py::test_numbers_beyond_a_c_int",
                "tests/test_f8_calls_without_module.py::test_sizes_of_other_integer_types")


@pytest.mark.gpu
def test_calls_without_the_module():
    run_without("-m", "gpu", "tests/test_gpu_f8_ops.py", "-k", "experts or by_index or tiles or another_device")


def test_numbers_beyond_a_c_int():
    """Refused by either way to make the calls; cut to 64 or 32 bits each would be a call that means something else."""
    import torch
    import __graft_entry__ as ge
    ge.build()
    import paper_1609_07061_b200.binding as q
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    x, bytes_, s = torch.zeros(64, 64, device=dev), torch.zeros(64, 64, dtype=torch.uint8, device=dev), torch.zeros(64, 16, dtype=torch.uint8, device=dev)
    c, i8 = bytes_.view(torch.float8_e4m3fn), bytes_.view(torch.int8)
    before = q.qnn_launch_count()
    for rows in (1 << 64, -(1 << 64), 1 << 63, (1 << 65) + 2):
        for call in (lambda: q.qnn_quantize_rows_i8(x, rows, 64, 64, i8, 64, x[0]), lambda: q.qnn_quantize_blocks_f8(x, rows, 64, 64, c, 64, s, 16),
                     lambda: q.qnn_quantize_tiles_f8(x, rows, 64, 64, c, 64, s, 16), lambda: q.qnn_quantize_columns_f8(x, rows, 16, 64, None, 1, c, 64, s, 16),
                     lambda: q.qnn_gemm_f8(c, 64, s, 16, c, 64, s, 16, rows, 4, 64, x, 64),
                     lambda: q.qnn_gemm_f8(c, 64, s, 16, c, 64, s, 16, 4, 4, 64, x, 64, b_transposed=rows),
                     lambda: q.qnn_gemm_f8_wgrad(c, 64, s, 16, c, 64, s, 16, None, 1, rows, 16, 16, x, 64)):
            with pytest.raises(OverflowError):
                call()
    assert q.qnn_launch_count() == before


def test_sizes_of_other_integer_types():
    """Sizes that are whole numbers without being ints, as the other per-token calls take them."""
    import numpy as np
    import torch
    import __graft_entry__ as ge
    ge.build()
    import paper_1609_07061_b200.binding as q
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    x, bytes_, s = torch.zeros(64, 64, device=dev), torch.zeros(64, 64, dtype=torch.uint8, device=dev), torch.zeros(64, 16, dtype=torch.uint8, device=dev)
    c, i8, off = bytes_.view(torch.float8_e4m3fn), bytes_.view(torch.int8), torch.zeros(3, dtype=torch.int64, device=dev)
    n = [np.int64(v) for v in range(65)]
    before = q.qnn_launch_count()
    q.qnn_quantize_rows_i8(x, n[0], n[64], n[64], i8, n[64], x[0])
    q.qnn_quantize_blocks_f8(x, n[0], n[64], n[64], c, n[64], s, n[16], index=off, src_rows=n[3], values=x, ld_values=n[64])
    q.qnn_quantize_tiles_f8(x, n[0], n[64], n[64], c, n[64], s, n[16], values=x, ld_values=n[64])
    q.qnn_quantize_columns_f8(x, n[0], n[16], n[64], off, n[2], c, n[64], s, n[16], values=x, ld_values=n[64])
    q.qnn_gemm_f8(c, n[64], s, n[16], c, n[64], s, n[16], n[0], n[4], n[64], x, n[64], bias=x[0], b_transposed=np.bool_(True))
    q.qnn_gemm_f8_grouped(c, n[64], s, n[16], c, n[64], s, n[16], off, n[2], n[0], n[4], n[64], x, n[64], bias=x[0])
    q.qnn_gemm_f8_wgrad(c, n[64], s, n[16], c, n[64], s, n[16], off, n[2], n[4], n[0], n[16], x, n[64])
    assert q.qnn_launch_count() == before
