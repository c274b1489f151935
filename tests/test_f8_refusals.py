"""Argument checks of the calls on 8-bit floating point: every refusal happens on the host, before anything is launched."""
import pytest
import torch

DEV = "cuda" if torch.cuda.is_available() else "cpu"
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def q():
    import __graft_entry__ as ge
    ge.build()
    import paper_1609_07061_b200.binding as b
    return b


def _mem(dtype=torch.float32, n=4096):
    # memory that is never read or written; 64-byte aligned, so that views have known alignment
    raw = torch.zeros(n * 8 + 64, dtype=torch.uint8, device=DEV)
    off = (-raw.data_ptr()) % 64
    return raw[off:off + n * torch.empty(0, dtype=dtype).element_size()].view(dtype)


def refuses(q, status, fn, *a, **kw):
    before = q.qnn_launch_count()
    with pytest.raises(q.QnnError) as e:
        fn(*a, **kw)
    assert e.value.status == status, (e.value.status, str(e.value))
    assert q.qnn_last_error() != "" and q.qnn_launch_count() == before


def test_quantisers_refuse(q):
    x, c, s, i = _mem(), _mem(E4M3), _mem(torch.uint8), _mem(torch.int64)
    INV, ALI, UNS = q.QNN_ERR_INVALID_ARG, q.QNN_ERR_ALIGNMENT, q.QNN_ERR_UNSUPPORTED
    rows, tiles = q.qnn_quantize_blocks_f8, q.qnn_quantize_tiles_f8
    cols = lambda x, r, K, ld, c, ldq, s, lds, **kw: q.qnn_quantize_columns_f8(x, r, K, ld, i, 2, c, ldq, s, lds, **kw)
    for f in (rows, tiles, cols):
        wide = 64 if f is cols else 16
        refuses(q, INV, f, x, -1, 64, 64, c, 64, s, wide)
        refuses(q, INV, f, x, 2, -64, 64, c, 64, s, wide)
        refuses(q, INV, f, x, 2, 64, 63, c, 64, s, wide)                       # ldx below K
        refuses(q, INV, f, x, 2, 65, 65, c, 64, s, 80)                         # ldq below K
        refuses(q, INV, f, None, 2, 64, 64, c, 64, s, wide)
        refuses(q, INV, f, x, 2, 64, 64, None, 64, s, wide)
        refuses(q, INV, f, x, 2, 64, 64, c, 64, None, wide)
        refuses(q, INV, f, x, 2, 64, 64, c, 64, s, 0)                          # no room for a row of scales
        refuses(q, INV, f, x, 2, 64, 64, c, 64, s, wide, values=x, ld_values=63)
        refuses(q, ALI, f, x, 2, 64, 64, c, 72, s, wide)
        refuses(q, ALI, f, x, 2, 64, 64, c[8:], 64, s, wide)
        refuses(q, ALI, f, x, 2, 64, 64, c, 64, s, wide + 8)
        refuses(q, ALI, f, x, 2, 64, 64, c, 64, s[4:], wide)
        refuses(q, UNS, f, x, (1 << 30) + 1, 64, 64, c, 64, s, wide)
        refuses(q, UNS, f, x, 1, (1 << 30) + 1, 1 << 31, c, 1 << 31, s, 1 << 31)
        with pytest.raises(TypeError):
            f(x.double(), 2, 64, 64, c, 64, s, wide)
        with pytest.raises(TypeError):
            f(x, 2, 64, 64, c.view(torch.int8), 64, s, wide)
        with pytest.raises(TypeError):
            f(x, 2, 64, 64, c, 64, s.view(torch.int8), wide)
        with pytest.raises(TypeError):
            f(x, 2, 64, 64, c, 64, s, wide, values=i, ld_values=64)
    refuses(q, INV, cols, x, 2, 64, 64, c, 64, s, 48)                          # scales: one a column
    for f in (tiles, cols):
        refuses(q, UNS, f, x, 65536 * 128, 64, 64, c, 64, s, 64)
    refuses(q, INV, rows, x, 2, 64, 64, c, 64, s, 16, index=i, src_rows=-1)
    with pytest.raises(TypeError):
        rows(x, 2, 64, 64, c, 64, s, 16, index=i.int(), src_rows=4)
    refuses(q, INV, q.qnn_quantize_columns_f8, x, 2, 64, 64, None, 2, c, 64, s, 64)
    refuses(q, INV, q.qnn_quantize_columns_f8, x, 2, 64, 64, i, -1, c, 64, s, 64)
    refuses(q, UNS, q.qnn_quantize_columns_f8, x, 2, 64, 64, i, q.QNN_F8_MAX_GROUPS + 1, c, 64, s, 64)
    # what the Python side cannot pass: pointers off their elements, unknown types
    f = q._lib.qnn_quantize_blocks_f8
    ptr = (x.data_ptr(), c.data_ptr(), s.data_ptr())
    assert f(ptr[0] + 2, 0, 2, 64, 64, None, 0, ptr[1], 0, 64, ptr[2], 16, None, 0, 0, None) == ALI
    assert f(ptr[0], 3, 2, 64, 64, None, 0, ptr[1], 0, 64, ptr[2], 16, None, 0, 0, None) == INV
    assert f(ptr[0], 0, 2, 64, 64, None, 0, ptr[1], 2, 64, ptr[2], 16, None, 0, 0, None) == INV
    assert f(ptr[0], 0, 2, 64, 64, None, 0, ptr[1], 0, 64, ptr[2], 16, ptr[0], 5, 64, None) == INV
    assert f(ptr[0], 0, 2, 64, 64, None, 0, ptr[1], 0, 64, ptr[2], 16, ptr[0] + 1, 1, 64, None) == ALI
    assert f(ptr[0], 0, 2, 64, 64, ptr[0] + 4, 9, ptr[1], 0, 64, ptr[2], 16, None, 0, 0, None) == ALI


def test_products_refuse(q):
    c, s, o, f, i = _mem(E4M3), _mem(torch.uint8), _mem(), _mem(), _mem(torch.int64)
    INV, ALI, UNS = q.QNN_ERR_INVALID_ARG, q.QNN_ERR_ALIGNMENT, q.QNN_ERR_UNSUPPORTED

    def dense(a=c, lda=64, sa=s, ldsa=16, b=c, ldb=64, sb=s, ldsb=16, M=4, N=4, K=64, out=o, ldo=4, **kw):
        q.qnn_gemm_f8(a, lda, sa, ldsa, b, ldb, sb, ldsb, M, N, K, out, ldo, **kw)

    def grouped(a=c, lda=64, sa=s, ldsa=16, b=c, ldb=64, sb=s, ldsb=16, M=4, N=4, K=64, out=o, ldo=4, offsets=i, groups=2, **kw):
        q.qnn_gemm_f8_grouped(a, lda, sa, ldsa, b, ldb, sb, ldsb, offsets, groups, M, N, K, out, ldo, **kw)

    def wgrad(a=c, lda=64, sa=s, ldsa=64, b=c, ldb=64, sb=s, ldsb=64, M=4, N=64, K=64, out=o, ldo=64, offsets=i, groups=2):
        q.qnn_gemm_f8_wgrad(a, lda, sa, ldsa, b, ldb, sb, ldsb, offsets, groups, M, N, K, out, ldo)

    for g in (dense, grouped, wgrad):
        for name in ("M", "N", "K"):
            refuses(q, INV, g, **{name: -1})
            refuses(q, UNS, g, **{name: (1 << 30) + 1})
        for name in ("a", "sa", "b", "sb", "out"):
            refuses(q, INV, g, **{name: None})
        for name in ("lda", "ldb"):
            refuses(q, INV, g, **{name: 48})
            refuses(q, ALI, g, **{name: 72})
            refuses(q, UNS, g, **{name: 1 << 40})
        for name in ("ldsa", "ldsb"):
            refuses(q, INV, g, **{name: 0})
            refuses(q, ALI, g, **{name: 72})
        refuses(q, ALI, g, a=c[8:])
        refuses(q, ALI, g, b=c[1:])
        refuses(q, ALI, g, sa=s[4:])
        refuses(q, ALI, g, sb=s[8:])
        refuses(q, INV, g, ldo=3)
        for bad in ({"a": c.view(torch.uint8)}, {"b": f}, {"sa": f}, {"sb": c}, {"out": i}, {"out": c}):
            with pytest.raises(TypeError):
                g(**bad)
    for g in (grouped, wgrad):
        refuses(q, INV, g, groups=-1)
        refuses(q, UNS, g, groups=q.QNN_F8_MAX_GROUPS + 1)
        refuses(q, INV, g, offsets=None)
        with pytest.raises(TypeError):
            g(offsets=i.int())
    refuses(q, UNS, grouped, ldb=1 << 39, N=100, ldo=100)                               # matrices of 2^40 bytes and more
    refuses(q, INV, dense, N=65, ldo=65, b_transposed=True)                    # weights read across have N elements a row
    for g in (dense, grouped):
        with pytest.raises(TypeError):
            g(bias=f.half())
        with pytest.raises(OverflowError):
            g(b_transposed=1 << 40)
        refuses(q, INV, g, b_transposed=2)
    refuses(q, UNS, dense, M=1 << 30, N=1 << 30, ldo=1 << 30)                  # more output tiles than are counted
    lib, p = q._lib, [t.data_ptr() for t in (c, s, o)]
    assert lib.qnn_gemm_f8(p[0], 2, 64, p[1], 16, p[0], 0, 64, p[1], 16, 0, None, 4, 4, 64, p[2], 0, 4, None) == INV
    assert lib.qnn_gemm_f8(p[0], 0, 64, p[1], 16, p[0], -1, 64, p[1], 16, 0, None, 4, 4, 64, p[2], 0, 4, None) == INV
    assert lib.qnn_gemm_f8(p[0], 0, 64, p[1], 16, p[0], 0, 64, p[1], 16, 0, None, 4, 4, 64, p[2], 4, 4, None) == INV
    assert lib.qnn_gemm_f8(p[0], 0, 64, p[1], 16, p[0], 0, 64, p[1], 16, 0, p[2] + 2, 4, 4, 64, p[2], 0, 4, None) == ALI
    assert lib.qnn_gemm_f8(p[0], 0, 64, p[1], 16, p[0], 0, 64, p[1], 16, 0, None, 4, 4, 64, p[2] + 2, 0, 4, None) == ALI


def test_empty_calls_are_ok(q):
    x, o = _mem(), _mem()
    before = q.qnn_launch_count()
    for rows, K in ((0, 64), (4, 0)):
        q.qnn_quantize_blocks_f8(x, rows, K, 64, None, 64, None, 16)
        q.qnn_quantize_tiles_f8(x, rows, K, 64, None, 64, None, 16)
        q.qnn_quantize_columns_f8(x, rows, K, 64, None, 1, None, 64, None, 64)
    for M, N in ((0, 4), (4, 0)):
        q.qnn_gemm_f8(None, 64, None, 16, None, 64, None, 16, M, N, 64, o, 4)
        q.qnn_gemm_f8_grouped(None, 64, None, 16, None, 64, None, 16, None, 2, M, N, 64, o, 4)
    q.qnn_gemm_f8_grouped(None, 64, None, 16, None, 64, None, 16, None, 0, 4, 4, 64, o, 4)
    q.qnn_gemm_f8_wgrad(None, 64, None, 64, None, 64, None, 64, None, 2, 4, 0, 64, o, 64)
    q.qnn_gemm_f8_wgrad(None, 64, None, 64, None, 64, None, 64, None, 2, 4, 64, 0, o, 64)
    assert q.qnn_launch_count() == before
