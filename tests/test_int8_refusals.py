"""Argument checks of the 8-bit language-model calls: every refusal happens on the host, before anything is launched."""
import pytest
import torch


@pytest.fixture(scope="module")
def q():
    import __graft_entry__ as ge
    ge.build()
    import paper_1609_07061_b200.binding as b
    return b


def _mem(n=4096, dtype=torch.float32):
    # CPU memory that is never dereferenced; 64-byte aligned, so that views have known alignment
    raw = torch.zeros(n * 8 + 64, dtype=torch.uint8)
    off = (-raw.data_ptr()) % 64
    return raw[off:off + n * torch.empty(0, dtype=dtype).element_size()].view(dtype)


def refuses(q, status, fn, *a, **kw):
    with pytest.raises(q.QnnError) as e:
        fn(*a, **kw)
    assert e.value.status == status, (e.value.status, str(e.value))
    assert q.qnn_last_error() != ""


def test_quantisers_refuse(q):
    x, c, s = _mem(), _mem(dtype=torch.int8), _mem()
    INV, ALI, UNS = q.QNN_ERR_INVALID_ARG, q.QNN_ERR_ALIGNMENT, q.QNN_ERR_UNSUPPORTED
    refuses(q, INV, q.qnn_quantize_rows_i8, x, -1, 64, 64, c, 64, s)
    refuses(q, INV, q.qnn_quantize_rows_i8, x, 2, 64, 63, c, 64, s)             # ldx below K
    refuses(q, INV, q.qnn_quantize_rows_i8, x, 2, 65, 65, c, 80, s)             # ldq below 96
    refuses(q, ALI, q.qnn_quantize_rows_i8, x, 2, 64, 64, c, 72, s)             # ldq not a multiple of 16
    refuses(q, ALI, q.qnn_quantize_rows_i8, x, 2, 64, 64, c[1:], 64, s)
    refuses(q, INV, q.qnn_quantize_rows_i8, None, 2, 64, 64, c, 64, s)
    refuses(q, INV, q.qnn_quantize_rows_i8, x, 2, 64, 64, c, 64, None)
    refuses(q, INV, q.qnn_quantize_rows_i8, x, 2, 64, 64, c, 64, s, values=x, ld_values=63)
    refuses(q, UNS, q.qnn_quantize_rows_i8, x, 1 << 31, 64, 64, c, 64, s)
    refuses(q, UNS, q.qnn_quantize_rows_i8, x, 1, (1 << 31) - 1, 1 << 31, c, 1 << 31, s)
    refuses(q, INV, q.qnn_rmsnorm_quant_i8, x, None, 2, 64, 64, 64, None, -1.0, c, 64, s)
    refuses(q, INV, q.qnn_rmsnorm_quant_i8, x, None, 2, 64, 64, 64, None, float("nan"), c, 64, s)
    refuses(q, INV, q.qnn_rmsnorm_quant_i8, x, x, 2, 64, 64, 63, None, 1e-5, c, 64, s)
    refuses(q, INV, q.qnn_rmsnorm_quant_i8, x, None, 2, 64, 64, 64, None, 1e-5, c, 64, s, sum_out=x, ld_sum=128)
    refuses(q, INV, q.qnn_rmsnorm_quant_i8, x, s, 2, 64, 64, 64, None, 1e-5, c, 64, s, sum_out=s, ld_sum=128)
    refuses(q, INV, q.qnn_silu_mul_quant_i8, x, None, 2, 64, 64, 64, c, 64, s)
    refuses(q, INV, q.qnn_silu_mul_quant_i8, x, x, 2, 64, 64, 60, c, 64, s)
    # a pointer that is not a multiple of its elements
    st = q._lib.qnn_quantize_rows_i8(x.data_ptr() + 2, q.QNN_TYPE_F32, 2, 64, 64, c.data_ptr(), 64, s.data_ptr(), None, 0, 0, None)
    assert st == ALI
    assert q._lib.qnn_quantize_rows_i8(x.data_ptr(), 7, 2, 64, 64, c.data_ptr(), 64, s.data_ptr(), None, 0, 0, None) == INV
    assert q._lib.qnn_quantize_rows_i8(x.data_ptr(), 0, 2, 64, 64, c.data_ptr(), 64, s.data_ptr(), x.data_ptr(), 9, 64, None) == INV
    # types that the C side could not tell apart
    with pytest.raises(TypeError):
        q.qnn_rmsnorm_quant_i8(x, x.bfloat16(), 2, 64, 64, 64, None, 1e-5, c, 64, s)
    with pytest.raises(TypeError):
        q.qnn_quantize_rows_i8(x.double(), 2, 64, 64, c, 64, s)
    with pytest.raises(TypeError):
        q.qnn_quantize_rows_i8(x, 2, 64, 64, c.to(torch.uint8), 64, s)


def test_product_refuses(q):
    a, s, o = _mem(dtype=torch.int8), _mem(), _mem()
    INV, ALI = q.QNN_ERR_INVALID_ARG, q.QNN_ERR_ALIGNMENT
    g = q.qnn_gemm_i8_scaled
    refuses(q, INV, g, a, 64, s, a, 64, s, -1, 4, 64, o, 4)
    refuses(q, q.QNN_ERR_OVERFLOW, g, a, 1 << 17, s, a, 1 << 17, s, 4, 4, 1 << 17, o, 4)
    refuses(q, q.QNN_ERR_UNSUPPORTED, g, a, 64, s, a, 64, s, (1 << 30) + 1, 4, 64, o, 4)
    refuses(q, INV, g, a, 64, None, a, 64, s, 4, 4, 64, o, 4)
    refuses(q, INV, g, None, 64, s, a, 64, s, 4, 4, 64, o, 4)
    refuses(q, INV, g, a, 48, s, a, 64, s, 4, 4, 64, o, 4)
    refuses(q, INV, g, a, 64, s, a, 64, s, 4, 4, 64, o, 3)
    refuses(q, ALI, g, a, 72, s, a, 64, s, 4, 4, 64, o, 4)
    refuses(q, ALI, g, a[8:], 64, s, a, 64, s, 4, 4, 64, o, 4)
    with pytest.raises(TypeError):
        g(a, 64, s, a, 64, s, 4, 4, 64, o.int(), 4)
    with pytest.raises(TypeError):
        g(a, 64, s.half(), a, 64, s, 4, 4, 64, o, 4)


def test_scores_refuse(q):
    z, f, i = _mem(), _mem(), _mem(dtype=torch.int64)
    INV, UNS = q.QNN_ERR_INVALID_ARG, q.QNN_ERR_UNSUPPORTED
    g = q.qnn_token_logprobs
    refuses(q, INV, g, z, -1, 10, 10, i, f)
    refuses(q, INV, g, z, 2, 0, 10, i, f)
    refuses(q, INV, g, z, 2, 10, 9, i, f)
    refuses(q, INV, g, z, 2, 10, 10, None, f)                                   # log probabilities of no tokens
    refuses(q, INV, g, z, 2, 10, 10, i, None)                                   # nothing asked for
    refuses(q, INV, g, z, 2, 10, 10, i, f, topk=11, top_ids=i)
    refuses(q, INV, g, z, 2, 10, 10, i, f, topk=2)
    refuses(q, INV, g, z, 2, 10, 10, i, f, topk=-1)
    refuses(q, UNS, g, z, 2, 100, 100, i, f, topk=33, top_ids=i)
    refuses(q, UNS, g, z, 2, 1 << 31, 1 << 31, i, f)
    refuses(q, INV, g, None, 2, 10, 10, i, f)
    b = q.qnn_token_logprobs_backward
    refuses(q, INV, b, z, 2, 10, 10, i, f, f, None, None, z, 10)
    refuses(q, INV, b, z, 2, 10, 10, None, f, f, f, None, z, 10)
    refuses(q, INV, b, z, 2, 10, 10, i, f, None, None, f, z, 10)
    refuses(q, INV, b, z, 2, 10, 10, i, None, f, f, None, z, 10)
    refuses(q, INV, b, z, 2, 10, 16, i, f, f, f, None, z, 10)                   # over the logits with another stride
    refuses(q, INV, b, z, 2, 10, 10, i, f, f, f, None, f, 9)
    with pytest.raises(TypeError):
        g(z, 2, 10, 10, i.int(), f)
    with pytest.raises(TypeError):
        b(z, 2, 10, 10, i, f, f, f, None, z.half(), 10)


def test_empty_calls_are_ok(q):
    q.qnn_quantize_rows_i8(None, 0, 64, 64, None, 64, None)
    q.qnn_rmsnorm_quant_i8(None, None, 0, 64, 64, 64, None, 1e-5, None, 64, None)
    q.qnn_silu_mul_quant_i8(None, None, 0, 64, 64, 64, None, 64, None)
    o = _mem()
    q.qnn_gemm_i8_scaled(None, 64, None, None, 64, None, 0, 4, 64, o, 4)
    q.qnn_gemm_i8_scaled(None, 64, None, None, 64, None, 4, 0, 64, o, 4)
    z = _mem()
    q.qnn_token_logprobs(z, 0, 10, 10, None, None)
    q.qnn_token_logprobs_backward(z, 0, 10, 10, None, None, None, None, None, z, 10)


def test_selftest_refuses(q):
    m = _mem(q.QNN_SELFTEST_CLUSTER_BYTES, torch.uint8)
    refuses(q, q.QNN_ERR_INVALID_ARG, q.qnn_selftest_cluster_timeout, 2, m)
    refuses(q, q.QNN_ERR_WORKSPACE, q.qnn_selftest_cluster_timeout, q.QNN_SELFTEST_PRODUCT, m[:-1])
    refuses(q, q.QNN_ERR_WORKSPACE, q.qnn_selftest_cluster_timeout, q.QNN_SELFTEST_SCORES, m[1:])
    refuses(q, q.QNN_ERR_WORKSPACE, q.qnn_selftest_cluster_timeout, q.QNN_SELFTEST_SCORES, None)
