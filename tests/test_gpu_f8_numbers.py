"""Products of 8-bit floating-point codes at the ends of codes, scales and sums, against the formula in 64 bits."""
import pytest
import torch

from test_gpu_f8_kernels import product
from test_gpu_f8_ops import B, E4M3, E5M2, TYPES, Operand, Out, gen, q, ref_blocks, up  # noqa: F401
from util import Guarded

pytestmark = pytest.mark.gpu


def same(got, want64):
    want = want64.to(torch.float32).to(got.dtype)
    return torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0, 1.0, -1.0), want.nan_to_num(0.0, 1.0, -1.0)) and \
        torch.equal(got.isinf(), want.isinf())


PAIRS = [(x, y) for x in (E4M3, E5M2) for y in (E4M3, E5M2)]


def all_bytes():
    return torch.arange(256, device="cuda").to(torch.uint8)


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("x_code,y_code", PAIRS)
def test_every_code_by_every_code(q, x_code, y_code, out):
    """One product a result, exact in fp32: all 256 bytes of either type, infinities and NaN among them, in every direction."""
    n = 256
    scale = torch.full((n, 256), 127, dtype=torch.uint8, device="cuda")
    for way in ("forward", "across", "gradient"):
        rows = {"forward": n, "across": 1, "gradient": 128}
        a = torch.zeros(128 if way == "gradient" else n, n if way == "gradient" else 16, dtype=torch.uint8, device="cuda")
        b = torch.zeros(n if way == "forward" else 128 if way == "gradient" else 16, 16 if way == "forward" else n, dtype=torch.uint8, device="cuda")
        if way == "gradient":
            a[0] = all_bytes()
        else:
            a[:, 0] = all_bytes()
        if way == "forward":
            b[:, 0] = all_bytes()
        else:
            b[0] = all_bytes()
        a, b = a.view(x_code), b.view(y_code)
        o = Guarded((n, n), out)
        if way == "gradient":
            q.qnn_gemm_f8_wgrad(a, n, scale, 256, b, n, scale, 256, None, 1, 1, n, n, o.t, n)
        else:
            q.qnn_gemm_f8(a, 16, scale, 256, b, b.shape[1], scale, 256, n, n, 1, o.t, n, b_transposed=way == "across")
        o.check()
        u, v = all_bytes().view(x_code).double(), all_bytes().view(y_code).double()
        assert same(o.t, u[:, None] * v[None]), way


ENDS = [(254, 0), (0, 254), (1, 253), (200, 60), (60, 200), (254, 100), (0, 0), (1, 1), (10, 110), (2, 100), (1, 126), (0, 127), (127, 0), (250, 126), (254, 126),
        (254, 254)]


@pytest.mark.parametrize("across", [False, True], ids=["forward", "across"])
@pytest.mark.parametrize("M,N,K", [(3, 130, 300), (7, 256, 1000), (300, 200, 2400), (2000, 640, 144), (2000, 2000, 600)])
def test_product_scales_at_the_ends(q, M, N, K, across):
    """All 2^(s - 127) of both operands together need be no fp32 numbers, only the sums.  One block of the reduction is not zero: whole
    numbers times one power of two.  Sums in fp32's normal range are exact.

    Below it: 32 terms are added to the sum at a time, in steps of 2^-25 of the largest power of two among them and the sum, whose exponent is
    -126 at least.  So each of the 32 loses less than 2^-151, the new sum, cut to fp32, less than 2^-149: 32 2^-151 + 2^-149 = 9 2^-149, four
    times for a block of 128: 36 2^-149.

    Above it a result is an infinity where the sum of magnitudes is no fp32 number, and never a NaN: partial sums may leave the range on
    either side."""
    g = gen(M + N + K)
    a = Operand(g, M, K, E4M3, (1, B), spread=0)
    w = Operand(g, K if across else N, N if across else K, E5M2, (B, B), spread=0)
    blk = up(K, B) // B // 2
    here = torch.zeros(K, dtype=torch.bool, device="cuda")
    here[blk * B:(blk + 1) * B] = True
    a.codes.view(torch.uint8)[:, :K][:, ~here] = 0
    av, wv = a.codes[:, :K].double(), w.codes[:, :N if across else K].double()
    other = wv if across else wv.t()
    sums, mags = av @ other, av.abs() @ other.abs()
    for sa, sw in ENDS:
        a.scale[:, blk] = sa
        w.scale[blk if across else slice(None), slice(None) if across else blk] = sw
        o = product(q, a, w, M, N, K, torch.float32, N, across)
        o.check()
        power = 2.0 ** (sa + sw - 254)
        want, most = sums * power, mags * power
        got = o.t.double()
        assert not got.isnan().any()
        fits = most < 2.0 ** 128
        assert got[fits].isfinite().all() and got[want.abs() >= 2.0 ** 128].isinf().all()
        lost = torch.where(got.isfinite(), (got - want).abs(), torch.zeros_like(got))
        assert (lost <= (0.0 if power >= 2.0 ** -126 else 36 * 2.0 ** -149)).all(), (sa, sw)


@pytest.mark.parametrize("M,N", [(1, 1), (300, 600), (2000, 2000)])
def test_sums_keep_25_bits_below_their_largest_term(q, M, N):
    """2^20 - 2^20 + a term 2^(20 - j), added in one step: what the two leave is the term, as long as it lies within 25 bits of them."""
    K = 640
    scale = torch.full((max(M, N), 16), 127, dtype=torch.uint8, device="cuda")
    for at in (0, 96, 500):
        for j in (3, 17, 24, 25):
            a, b = torch.zeros(M, K, device="cuda"), torch.zeros(N, K, device="cuda")
            a[:, at], b[:, at] = 2.0 ** 10, 2.0 ** 10
            a[:, at + 7], b[:, at + 7] = -(2.0 ** 10), 2.0 ** 10
            a[:, at + 12], b[:, at + 12] = 2.0 ** ((20 - j) // 2), 2.0 ** (20 - j - (20 - j) // 2)
            o = Guarded((M, N), torch.float32)
            q.qnn_gemm_f8(a.to(E5M2), K, scale, 16, b.to(E5M2), K, scale, 16, M, N, K, o.t, N)
            o.check()
            assert (o.t == 2.0 ** (20 - j)).all(), (at, j)


@pytest.mark.parametrize("dtype", TYPES[1:])
@pytest.mark.parametrize("code", [E4M3, E5M2])
def test_quantisers_at_the_ends_of_16_bit_types(q, code, dtype):
    """Zeros, the least subnormal, the largest number, infinities and NaN of the type, each in a block of its own."""
    info = torch.finfo(dtype)
    tiny = info.smallest_normal * info.eps
    rows = [[0.0], [-0.0], [tiny], [-tiny, tiny * 3], [info.smallest_normal], [info.max, 1.0], [-info.max, info.max / 2], [float("inf"), 1.0],
            [1.0, float("-inf")], [float("nan"), 2.0], [info.max, float("nan")], [17.0, 19.0, 448.0], [1.75, 1.0], [1.75 + 2 * info.eps, 1.0]]
    t = torch.zeros(len(rows), B, device="cuda", dtype=dtype)
    for i, r in enumerate(rows):
        t[i, :len(r)] = torch.tensor(r, dtype=torch.float64).to(dtype)
    o = Out(len(rows), B, len(rows), 1, code, torch.float32)
    q.qnn_quantize_blocks_f8(t, len(rows), B, B, o.q, o.ldq, o.scale.t, o.lds, values=o.values.t, ld_values=o.ldv)
    o.check(*ref_blocks(t.double(), 1, B, code), (1, B))
    assert (o.scale.t[:, 0] == 255).tolist() == [not torch.tensor(r).isfinite().all() for r in rows]
    cols = t.t().contiguous()
    o = Out(2 * B, len(rows), 2, len(rows), code, torch.float32)
    q.qnn_quantize_columns_f8(cols, B, len(rows), len(rows), None, 1, o.q, o.ldq, o.scale.t, o.lds, values=o.values.t, ld_values=o.ldv)
    o.check(*ref_blocks(cols.double(), B, 1, code), (B, 1), rows=B)
    for i in range(len(rows)):
        o = Out(1, B, 1, 1, code, torch.float32)
        q.qnn_quantize_tiles_f8(t[i:i + 1], 1, B, B, o.q, o.ldq, o.scale.t, o.lds, values=o.values.t, ld_values=o.ldv)
        o.check(*ref_blocks(t[i:i + 1].double(), B, B, code), (B, B))
