"""The 8-bit language-model calls against plain formulas in 64 bits.

Tolerances.  U = 2^-24 is half a unit in the last place of fp32.  Quantisers: a sum of squares over at most ~130 terms a
thread and a tree of ~20 is off by at most 150 U relative, its square root by half of that, exp and the division of the gate
by (|a| + 8) U: scales within 2e-5 relative, and t * 127 / max within 127 * 2e-5 < 3e-3 of the exact number before it is
rounded.  Product: int32 sum exact, three fp32 roundings.  Scores: a thread adds up to V / 128 terms, each exp off by
(|x| + 4) U where it matters little (|x| large).  16-bit results of the product and the gradient are the fp32 results of the
same call rounded once, bit for bit, so only the fp32 results are held to a tolerance.
"""
import numpy as np
import pytest
import torch

from util import Guarded

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def q():
    import paper_1609_07061_b200.binding as b
    return b


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def strided(rows, K, ld, dtype, offset=0, g=None, scale=1.0):
    """[rows, K] view with row stride ld, `offset` elements into its buffer; the rest of the buffer is NaN."""
    buf = torch.full((offset + rows * ld + 16,), float("nan"), dtype=dtype, device="cuda")
    v = buf[offset:offset + rows * ld].view(rows, ld)[:, :K]
    v.copy_((torch.randn(rows, K, generator=g, device="cuda") * scale).to(dtype))
    return v


def pad32(K):
    return (K + 31) // 32 * 32


class Quantised:
    """Guarded outputs of a quantising call, and the checks they all share."""

    def __init__(self, rows, K, ldq=None, values=None, ld_values=None):
        self.rows, self.K = rows, K
        self.ldq = ldq or (pad32(K) + 16)
        self.codes = Guarded((rows, self.ldq), torch.int8)
        self.scale = Guarded((rows,), torch.float32)
        self.ldv = ld_values or K
        self.values = Guarded((rows, self.ldv), values) if values else None

    def check(self, t64, rows_ok=None):
        """t64: the exact rows.  rows_ok: rows with finite, non-zero values."""
        for b in (self.codes, self.scale, self.values):
            if b is not None:
                b.check()
        codes, scale = self.codes.t, self.scale.t
        assert (codes[:, self.K:pad32(self.K)] == 0).all(), "pads up to the next 32 are zero"
        left = codes[:, pad32(self.K):].contiguous().view(torch.uint8)
        assert (left == 0xA5).all(), "bytes past the pads are untouched"
        top = t64.abs().amax(1)
        rel = ((scale.double() - top / 127) / (top / 127)).abs().max().item()
        assert rel < 2e-5, rel
        off = (codes[:, :self.K].double() - t64 * (127 / top)[:, None]).abs().max().item()
        assert off <= 0.5 + 3e-3, off
        assert codes[:, :self.K].abs().amax(1).min().item() == 127
        if self.values is not None:
            want = (codes[:, :self.K].float() * scale[:, None]).to(self.values.dtype)
            assert torch.equal(self.values.t[:, :self.K], want)


SHAPES = [(1, 1), (3, 2), (1, 7), (5, 31), (2, 32), (9, 33), (4, 100), (7, 255), (3, 256), (33, 1000), (2, 4095), (1, 4096), (1, 4097),
          (301, 640), (2, 8192), (300, 8193), (1, 11000), (2, 16384), (1, 16385), (3, 32768), (2, 32769), (1, 40003)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", SHAPES)
def test_quantize_rows(q, rows, K, dtype):
    g = gen(rows * 7 + K)
    # dense; padded and aligned; rows of even offset; rows of odd offset
    for n, (ld, off) in enumerate([(K, 0), ((K + 7) // 8 * 8 + 8, 0), ((K + 1) // 2 * 2, 2), (K + 3, 1)]):
        x = strided(rows, K, ld, dtype, off, g, 3.0)
        o = Quantised(rows, K, values=TYPES[n % 3], ld_values=K + (n % 2))
        q.qnn_quantize_rows_i8(x, rows, K, ld, o.codes.t, o.ldq, o.scale.t, values=o.values.t, ld_values=o.ldv)
        o.check(x.double())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", SHAPES)
def test_rmsnorm_quant(q, rows, K, dtype):
    g = gen(rows * 11 + K)
    eps = 1e-5
    for n, (ld, off) in enumerate([(K, 0), ((K + 7) // 8 * 8 + 8, 0), ((K + 1) // 2 * 2, 2), (K + 3, 1)]):
        x = strided(rows, K, ld, dtype, off, g, 2.0)
        r = strided(rows, K, ld, dtype, off, g, 5.0) if n != 1 else None
        gamma = (1 + 0.3 * torch.randn(K, generator=g, device="cuda")).to(dtype) if n != 2 else None
        o = Quantised(rows, K, values=dtype if n != 3 else None)
        s = Guarded((rows, ld), dtype) if n != 1 else None
        s64 = x.double() + (r.double() if r is not None else 0)
        t64 = s64 / torch.sqrt((s64 * s64).mean(1, keepdim=True) + eps) * (gamma.double() if gamma is not None else 1)
        want_sum = (x.float() + (r.float() if r is not None else 0)).to(dtype)
        q.qnn_rmsnorm_quant_i8(x, r, rows, K, ld, ld, gamma, eps, o.codes.t, o.ldq, o.scale.t, sum_out=s.t if s else None, ld_sum=ld,
                               values=o.values.t if o.values else None, ld_values=o.ldv)
        o.check(t64)
        if s:
            s.check()
            assert torch.equal(s.t[:, :K], want_sum)


@pytest.mark.parametrize("K", [64, 1000, 4099, 33000])
@pytest.mark.parametrize("over", ["x", "residual"])
def test_rmsnorm_sum_in_place(q, K, over):
    g = gen(K)
    for dtype in TYPES:
        x, r = strided(5, K, K, dtype, 0, g), strided(5, K, K, dtype, 0, g)
        want = Quantised(5, K)
        s = torch.empty(5, K, dtype=dtype, device="cuda")
        q.qnn_rmsnorm_quant_i8(x, r, 5, K, K, K, None, 1e-6, want.codes.t, want.ldq, want.scale.t, sum_out=s, ld_sum=K)
        got = Quantised(5, K)
        into = x if over == "x" else r
        q.qnn_rmsnorm_quant_i8(x, r, 5, K, K, K, None, 1e-6, got.codes.t, got.ldq, got.scale.t, sum_out=into, ld_sum=K)
        assert torch.equal(into, s)
        assert torch.equal(got.codes.t, want.codes.t) and torch.equal(got.scale.t, want.scale.t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", SHAPES)
def test_silu_mul_quant(q, rows, K, dtype):
    g = gen(rows * 13 + K)
    for n, ld in enumerate([2 * K, (2 * K + 15) // 8 * 8, 2 * K + 1]):
        both = strided(rows, 2 * K, ld, dtype, 0, g, 4.0)
        gate, up = both[:, :K], both[:, K:]
        o = Quantised(rows, K, values=dtype)
        q.qnn_silu_mul_quant_i8(gate, up, rows, K, ld, ld, o.codes.t, o.ldq, o.scale.t, values=o.values.t, ld_values=o.ldv)
        a = gate.double()
        o.check(a / (1 + torch.exp(-a)) * up.double())


@pytest.mark.parametrize("K", [1, 96, 4097, 40000])
def test_quantisers_special_rows(q, K):
    """Zero rows, rows too small to scale, infinities and NaN, squares that overflow, large gates."""
    inf, nan = float("inf"), float("nan")
    x = torch.randn(8, K, generator=gen(K), device="cuda")
    x[0] = 0.0
    x[1] = 1e-37
    x[2, K // 2] = inf
    x[3, K - 1] = nan
    x[4, 0] = -inf
    x[5] = 2e38
    x[6] = 1e-30
    o = Quantised(8, K, values=torch.float32)
    q.qnn_quantize_rows_i8(x, 8, K, K, o.codes.t, o.ldq, o.scale.t, values=o.values.t, ld_values=K)
    c, s, v = o.codes.t[:, :K], o.scale.t, o.values.t
    assert s[:2].tolist() == [0.0, 0.0] and (c[:2] == 0).all() and (v[:2] == 0).all()
    assert s[2:5].isnan().all() and (c[2:5] == 0).all() and v[2:5].isnan().all()
    assert (c[5:7] == 127).all() and s[5:].isfinite().all()
    o = Quantised(8, K, values=torch.float32)
    q.qnn_rmsnorm_quant_i8(x, None, 8, K, K, K, None, 0.0, o.codes.t, o.ldq, o.scale.t, values=o.values.t, ld_values=K)
    c, s = o.codes.t[:, :K], o.scale.t
    assert s[:2].tolist() == [0.0, 0.0] and (c[:2] == 0).all() and (o.values.t[:2] == 0).all()
    assert s[2:6].isnan().all() and (c[2:6] == 0).all()          # 2e38 squared is past fp32
    up = torch.ones(8, K, device="cuda")
    gate = x.clone()
    gate[5] = 90.0
    gate[6] = -200.0
    gate[7] = 20.0
    o = Quantised(8, K)
    q.qnn_silu_mul_quant_i8(gate, up, 8, K, K, K, o.codes.t, o.ldq, o.scale.t)
    c, s = o.codes.t[:, :K], o.scale.t
    assert s[2:5].isnan().all() and (c[2:5] == 0).all()
    assert s[6].item() == 0.0 and (c[6] == 0).all()
    assert (c[5] == 127).all() and abs(s[5].item() - 90 / 127) < 1e-5
    assert (c[7] == 127).all()


def product_want(a, b, sa, sb, bias, K):
    y = (a[:, :K].double() @ b[:, :K].double().t())
    mag = (y * sa.double()[:, None] * sb.double()[None, :])
    return mag + (bias.double()[None, :] if bias is not None else 0), mag.abs()


def check_product(q, M, N, K, dtype, bias=True, ldo=None, offset=0, lda=None, seed=0):
    g = gen(seed + M * 31 + N * 7 + K)
    lda = lda or (K + 15) // 16 * 16
    ldb = (K + 15) // 16 * 16 + 32
    # bytes past K are garbage: they must not reach the sum
    a = torch.randint(-128, 128, (M, lda), generator=g, device="cuda", dtype=torch.int8)
    b = torch.randint(-128, 128, (N, ldb), generator=g, device="cuda", dtype=torch.int8)
    sa = torch.rand(M, generator=g, device="cuda") + 0.5
    sb = (torch.rand(N, generator=g, device="cuda") + 0.5) / 1000
    bi = torch.randn(N, generator=g, device="cuda") if bias else None
    ldo = ldo or N
    out = Guarded((M * ldo + offset,), dtype)
    view = out.t[offset:].view(M, ldo)
    q.qnn_gemm_i8_scaled(a, lda, sa, b, ldb, sb, M, N, K, view, ldo, bias=bi)
    out.check()
    if dtype == torch.float32:
        want, mag = product_want(a, b, sa, sb, bi, K)
        bad = (view[:, :N].double() - want).abs() > 3 * U * mag + U * want.abs()
    else:
        full = torch.empty(M, N, device="cuda")
        q.qnn_gemm_i8_scaled(a, lda, sa, b, ldb, sb, M, N, K, full, N, bias=bi)
        bad = view[:, :N] != full.to(dtype)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())
    if ldo > N:
        left = view[:, N:].contiguous().view(torch.uint8)
        assert (left == 0xA5).all()


PRODUCTS = [(1, 1, 1), (1, 128, 128), (1, 4096, 4096), (2, 31, 17), (3, 129, 1000), (8, 2048, 512), (16, 300, 4096), (17, 257, 385), (32, 64, 96),
            (33, 1000, 777), (64, 4096, 128), (65, 96, 2048), (100, 4096, 4096), (127, 515, 130), (128, 128, 16384), (129, 128, 128),
            (200, 1000, 333), (256, 256, 4096), (300, 2047, 1111), (701, 2047, 1111), (1000, 4096, 64), (2500, 2304, 520), (4096, 4100, 200),
            (3000, 8192, 257), (10000, 33, 160)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(q, M, N, K, dtype):
    check_product(q, M, N, K, dtype, bias=(M + N) % 2 == 0)
    assert q.qnn_device_status() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(5, 130, 200), (130, 260, 300), (2500, 2304, 300)])
def test_product_output_strides(q, M, N, K, dtype):
    for ldo, offset in [(N + 8, 0), (N + 1, 0), (N, 1), (N + 16, 8)]:
        check_product(q, M, N, K, dtype, ldo=ldo, offset=offset, lda=(K + 15) // 16 * 16 + 64)


@pytest.mark.parametrize("M,N", [(1, 5), (20, 40), (300, 200)])
def test_product_largest_sums(q, M, N):
    """The longest K with every product 2^14: the int32 sum is 2^31 - 2^14."""
    K = (1 << 17) - 1
    a = torch.full((M, 1 << 17), -128, dtype=torch.int8, device="cuda")
    b = torch.full((N, 1 << 17), -128, dtype=torch.int8, device="cuda")
    b[1:2] = 127
    one = torch.ones(max(M, N), device="cuda")
    out = torch.empty(M, N, device="cuda")
    q.qnn_gemm_i8_scaled(a, 1 << 17, one, b, 1 << 17, one, M, N, K, out, N)
    want = torch.full((M, N), float(K * 16384), dtype=torch.float64, device="cuda")
    want[:, 1:2] = -float(K * 128 * 127)
    assert torch.equal(out, want.float())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", [(1, 257), (3, 300), (2, 1031), (5, 4099), (301, 519), (2, 9001), (400, 2051)])
def test_quantisers_tensors_at_different_offsets(q, rows, K, dtype):
    """Every tensor starts elsewhere in its 16 bytes, and so does every row; the outputs are those of aligned tensors, bit for bit,
    and nothing beside the rows is written."""
    g = gen(rows + K)
    wide = (K + 15) // 8 * 8

    def at(off, ld):
        return torch.full((rows * ld + 16,), 7.0, dtype=dtype, device="cuda")[off:off + rows * ld].view(rows, ld)

    x, r = (torch.randn(rows, wide, generator=g, device="cuda").to(dtype) for _ in range(2))
    gamma = (1 + 0.3 * torch.randn(wide, generator=g, device="cuda")).to(dtype)
    x2, r2, s2 = at(1, K), at(3, K + 2), at(5, K + 1)
    x2.copy_(x[:, :K]); r2[:, :K].copy_(r[:, :K])
    gamma2 = torch.empty(wide + 8, dtype=dtype, device="cuda")[7:7 + K]
    gamma2.copy_(gamma[:K])
    for vt in TYPES:
        one, two = Quantised(rows, K, values=vt, ld_values=wide), Quantised(rows, K, values=vt, ld_values=K + 3)
        total = torch.empty(rows, wide, dtype=dtype, device="cuda")
        q.qnn_rmsnorm_quant_i8(x, r, rows, K, wide, wide, gamma, 1e-5, one.codes.t, one.ldq, one.scale.t, sum_out=total, ld_sum=wide,
                               values=one.values.t, ld_values=one.ldv)
        q.qnn_rmsnorm_quant_i8(x2, r2, rows, K, K, K + 2, gamma2, 1e-5, two.codes.t, two.ldq, two.scale.t, sum_out=s2, ld_sum=K + 1,
                               values=two.values.t, ld_values=two.ldv)
        assert torch.equal(s2[:, :K], total[:, :K]) and (s2[:, K:] == 7).all()
        top = one.codes.t[:, :K].int() - two.codes.t[:, :K].int()
        # (the sum of squares is added in another order, which moves the scale by roundings, not the codes)
        assert not top.any()
        assert ((one.scale.t - two.scale.t).abs() <= 1e-5 * one.scale.t).all()
        # in place: over x, and over the residual
        for over, ld in ((0, K), (1, K + 2)):
            a, b = x2.clone(), r2.clone()
            o = Quantised(rows, K, values=vt, ld_values=K + 3)
            q.qnn_rmsnorm_quant_i8(a, b, rows, K, K, K + 2, gamma2, 1e-5, o.codes.t, o.ldq, o.scale.t, sum_out=(a, b)[over], ld_sum=ld,
                                   values=o.values.t, ld_values=o.ldv)
            assert torch.equal((a, b)[over][:, :K], total[:, :K]) and torch.equal(o.codes.t, two.codes.t)
        one, two = Quantised(rows, K, values=vt, ld_values=wide), Quantised(rows, K, values=vt, ld_values=K + 3)
        q.qnn_silu_mul_quant_i8(x, r, rows, K, wide, wide, one.codes.t, one.ldq, one.scale.t, values=one.values.t, ld_values=one.ldv)
        q.qnn_silu_mul_quant_i8(x2, r2, rows, K, K, K + 2, two.codes.t, two.ldq, two.scale.t, values=two.values.t, ld_values=two.ldv)
        assert torch.equal(one.codes.t, two.codes.t) and torch.equal(one.scale.t, two.scale.t)
        assert torch.equal(one.values.t[:, :K], two.values.t[:, :K])


def test_quantisers_without_k_give_scale_zero(q):
    c = torch.full((5, 32), 7, dtype=torch.int8, device="cuda")
    x = torch.ones(5, 32, device="cuda")
    for call in (lambda s: q.qnn_quantize_rows_i8(x, 5, 0, 32, c, 32, s), lambda s: q.qnn_rmsnorm_quant_i8(x, None, 5, 0, 32, 32, None, 0.0, c, 32, s),
                 lambda s: q.qnn_silu_mul_quant_i8(x, x, 5, 0, 32, 32, c, 32, s)):
        s = torch.full((6,), 3.0, device="cuda")
        call(s)
        assert s.tolist() == [0.0] * 5 + [3.0] and (c == 7).all()


def test_product_without_k_is_the_bias(q):
    for dtype in TYPES:
        s, bias = torch.ones(64, device="cuda"), torch.randn(50, device="cuda")
        out = torch.full((3, 50), 7.0, dtype=dtype, device="cuda")
        q.qnn_gemm_i8_scaled(None, 0, s, None, 0, s, 3, 50, 0, out, 50, bias=bias)
        assert torch.equal(out, bias.to(dtype).expand(3, 50))
        q.qnn_gemm_i8_scaled(None, 0, s, None, 0, s, 3, 50, 0, out, 50)
        assert (out == 0).all()


def test_product_nan_scale_stays_in_its_row(q):
    """A row whose quantiser saw a NaN has a NaN scale: its outputs are NaN, no other row's are."""
    for M in (4, 200):
        a = torch.randint(-127, 128, (M, 128), device="cuda", dtype=torch.int8)
        b = torch.randint(-127, 128, (96, 128), device="cuda", dtype=torch.int8)
        sa, sb = torch.ones(M, device="cuda"), torch.ones(96, device="cuda")
        sa[2] = float("nan")
        out = torch.empty(M, 96, dtype=torch.bfloat16, device="cuda")
        q.qnn_gemm_i8_scaled(a, 128, sa, b, 128, sb, M, 96, 128, out, 96)
        n = out.isnan().all(1)
        assert n[2] and not out.isnan().any(1)[torch.arange(M, device="cuda") != 2].any()


# ---- scores ------------------------------------------------------------------------------------------------------

def run_scores(q, z, ids, topk, ldl):
    T, V = z.shape
    lp, h, lse = (Guarded((T,), torch.float32) for _ in range(3))
    tl, ti = (Guarded((T, topk), torch.float32), Guarded((T, topk), torch.int64)) if topk else (None, None)
    q.qnn_token_logprobs(z, T, V, ldl, ids, lp.t, entropy=h.t, lse=lse.t, topk=topk, top_logprob=tl.t if topk else None,
                         top_ids=ti.t if topk else None)
    for b in (lp, h, lse, tl, ti):
        if b is not None:
            b.check()
    return lp.t, h.t, lse.t, (tl.t if topk else None), (ti.t if topk else None)


def check_scores(q, z, ids, topk, ldl):
    T, V = z.shape
    lp, h, lse, tl, ti = run_scores(q, z, ids, topk, ldl)
    z64 = z.double()
    logp = torch.log_softmax(z64, 1)
    p = logp.exp()
    h64 = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    lse64 = torch.logsumexp(z64, 1)
    big = z64.masked_fill(z64 == float("-inf"), 0).abs().amax(1)
    tol = (V / 128 + 64) * U + 4 * U * big
    assert ((lse.double() - lse64).abs() <= tol).all(), (lse.double() - lse64).abs().max()
    assert ((h.double() - h64).abs() <= 4 * tol * (1 + h64)).all(), (h.double() - h64).abs().max()
    inside = (ids >= 0) & (ids < V)
    want = logp.gather(1, ids.clamp(0, V - 1)[:, None])[:, 0]
    fin = inside & want.isfinite()
    assert ((lp.double() - want).abs()[fin] <= (tol + 4 * U * want.abs())[fin]).all()
    assert (lp[inside & ~want.isfinite()] == float("-inf")).all()
    assert (lp[~inside] == 0).all()
    if topk:
        order = torch.sort(z64, dim=1, descending=True, stable=True).indices[:, :topk]
        assert torch.equal(ti, order), (ti != order).nonzero()[:5].tolist()
        w = logp.gather(1, order)
        f = w.isfinite()
        assert ((tl.double() - w).abs()[f] <= (tol[:, None] + 4 * U * w.abs().nan_to_num(0, 0, 0))[f]).all()
        assert (tl[~f] == float("-inf")).all()


SCORES = [(1, 1, 1), (3, 2, 2), (2, 7, 5), (5, 40, 20), (4, 333, 32), (130, 1000, 5), (3, 4095, 8), (2, 4104, 1), (700, 5000, 0), (33, 50021, 5),
          (1, 128000, 20), (4, 128001, 5), (320, 32000, 8), (2, 300001, 32)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,topk", SCORES)
def test_scores(q, T, V, topk, dtype):
    g = gen(T + V)
    for n, (ld, off) in enumerate([(V, 0), (V + 5, 3)]):
        z = strided(T, V, ld, dtype, off, g, 3.0)
        if n and V > 10:
            z[:, V // 2:V // 2 + V // 5] = float("-inf")
            z[:, 1] = torch.finfo(dtype).min
        ids = torch.randint(0, V, (T,), generator=g, device="cuda")
        if T > 2:
            ids[0], ids[1] = -1, V
        check_scores(q, z, ids, topk, ld)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [50, 3000, 20001, 70000])
def test_scores_masks_and_ties(q, V, dtype):
    """Equal logits in masses, rows with fewer entries left than alternatives, masks of the type's lowest value, wide ranges."""
    inf = float("inf")
    z = torch.randn(9, V, generator=gen(V), device="cuda").to(dtype)
    z[0] = 2.5                                           # all equal
    z[1] = -inf
    z[1, [V - 1, 3, V // 2]] = torch.tensor([1.0, 1.0, 3.0], device="cuda", dtype=dtype)   # three left, two of them equal
    z[2] = torch.finfo(dtype).min                        # all masked by the lowest value: uniform
    z[3] = torch.finfo(dtype).min
    z[3, 7] = 0.0
    z[4, ::2] = 4.0                                      # half of the row ties at the top
    z[5] = -inf
    z[5, V - 1] = -30000.0                               # one entry left
    z[6] *= 5000.0                                       # one entry takes all the probability
    z[7, 10] = -0.0
    z[7, 9] = 0.0
    z[8, :] = torch.where(z[8] > 0, -z[8], z[8])
    z[8, 20], z[8, 30] = -0.0, 0.0                       # signed zeros tie at the top
    ids = torch.tensor([5, 3, 0, 7, 1, V - 1, 4, 9, 30], device="cuda")
    check_scores(q, z, ids, 8, V)


def test_scores_rows_with_nothing_left_and_bad_rows(q):
    inf, nan = float("inf"), float("nan")
    for dtype in TYPES:
        for V in (64, 9000, 70001):
            z = torch.randn(4, V, generator=gen(V), device="cuda").to(dtype)
            z[0] = -inf
            z[1, V - 2] = nan
            z[2, 11] = inf
            ids = torch.tensor([5, 3, 2, 1], device="cuda")
            lp, h, lse, tl, ti = run_scores(q, z, ids, 4, V)
            assert lse[0].item() == -inf and lp[0].item() == -inf and h[0].item() == 0.0 and (tl[0] == -inf).all()
            assert ti[0].tolist() == [0, 1, 2, 3]
            for r in (1, 2):
                assert lse[r].isnan() and lp[r].isnan() and h[r].isnan() and tl[r].isnan().all()
                assert ((ti[r] >= 0) & (ti[r] < V)).all()
            assert ti[1, 0].item() == V - 2 and ti[2, 0].item() == 11
            assert lse[3].isfinite()


def grad_want(z64, ids, gl, gh):
    """The gradient by 64-bit autograd of the definition."""
    V = z64.shape[1]
    z = z64.clone().requires_grad_(True)
    logp = torch.log_softmax(z, 1)
    p = logp.exp()
    h = -(torch.where(p > 0, p * logp.masked_fill(p == 0, 0), torch.zeros_like(p))).sum(1)
    total = z.sum() * 0 if z64.isfinite().all() else 0
    if gl is not None:
        inside = (ids >= 0) & (ids < V)
        total = total + (logp.gather(1, ids.clamp(0, V - 1)[:, None])[:, 0] * gl.double() * inside).sum()
    if gh is not None:
        total = total + (h * gh.double()).sum()
    (d,) = torch.autograd.grad(total, z)
    return d


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(1, 1), (3, 2), (2, 7), (5, 333), (130, 1000), (3, 50021), (2, 128000)])
def test_scores_gradient(q, T, V, dtype):
    g = gen(T * 3 + V)
    for n, (ld, off, ldd, offd) in enumerate([(V, 0, V, 0), (V + 5, 3, V + 5, 3), (V + 3, 1, V + 8, 2)]):
        z = strided(T, V, ld, dtype, off, g, 3.0)
        ids = torch.randint(0, V, (T,), generator=g, device="cuda")
        if T > 2:
            ids[1] = -100
        z64 = z.double()
        lse64 = torch.logsumexp(z64, 1)
        p = (z64 - lse64[:, None]).exp()
        h64 = -torch.where(p > 0, p * (z64 - lse64[:, None]), torch.zeros_like(p)).sum(1)
        gl = torch.randn(T, generator=g, device="cuda") if n != 2 else None
        gh = torch.randn(T, generator=g, device="cuda") if n != 1 else None
        d = Guarded((T * ldd + offd,), dtype)
        view = d.t[offd:].view(T, ldd)
        q.qnn_token_logprobs_backward(z, T, V, ld, ids, lse64.float(), h64.float(), gl, gh, view, ldd)
        d.check()
        if ldd > V:
            assert (view[:T - 1, V:].contiguous().view(torch.uint8) == 0xA5).all()
        if dtype != torch.float32:
            full = torch.empty(T, V, device="cuda")
            q.qnn_token_logprobs_backward(z.float().contiguous(), T, V, V, ids, lse64.float(), h64.float(), gl, gh, full, V)
            assert torch.equal(view[:, :V], full.to(dtype)), n
            continue
        want = grad_want(z64, ids, gl, gh)
        # p is off by (|z| + |lse| + 4) 2 U relative, the entropy by U of itself; one rounding to the type
        a = gl.double().abs()[:, None] if gl is not None else 0
        b = gh.double().abs()[:, None] if gh is not None else 0
        terms = p * (a + b * ((z64 - lse64[:, None]).abs() + h64[:, None] + 1))
        tol = terms * 2 * U * (z64.abs() + lse64.abs()[:, None] + 8) + 3 * U * want.abs() + 2 * U * a * p + 1e-37
        hot = torch.zeros_like(p)
        hot.scatter_(1, ids.clamp(0, V - 1)[:, None], 1.0)
        tol = tol + hot * a * 2 * U
        bad = (view[:, :V].double() - want).abs() > tol
        assert not bad.any(), (n, int(bad.sum()), bad.nonzero()[:4].tolist())


def test_scores_gradient_against_differences(q):
    """<gradient, direction> against central differences of the definition in 64 bits."""
    T, V = 6, 700
    g = gen(3)
    z = torch.randn(T, V, generator=g, device="cuda") * 2
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    gl, gh = torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
    lp, h, lse = (torch.empty(T, device="cuda") for _ in range(3))
    q.qnn_token_logprobs(z, T, V, V, ids, lp, entropy=h, lse=lse)
    d = torch.empty_like(z)
    q.qnn_token_logprobs_backward(z, T, V, V, ids, lse, h, gl, gh, d, V)

    def f(x):
        logp = torch.log_softmax(x, 1)
        return (logp.gather(1, ids[:, None])[:, 0] * gl.double()).sum() - ((logp.exp() * logp).sum(1) * gh.double()).sum()
    for k in range(8):
        u = torch.randn(T, V, generator=g, device="cuda").double()
        if k < 2:                                        # the tokens' own entries
            u = torch.zeros_like(u).scatter_(1, ids[:, None], 1.0)
        step = 1e-5
        diff = (f(z.double() + step * u) - f(z.double() - step * u)) / (2 * step)
        got = (d.double() * u).sum()
        # differences: third derivatives times step^2 and 1e-16 / step; the gradient: fp32
        assert abs((got - diff).item()) <= 1e-5 * (1 + (d.double() * u).abs().sum().item())


def test_scores_gradient_masked_and_in_place(q):
    inf = float("-inf")
    for dtype in TYPES:
        for V in (100, 5001):
            z = torch.randn(4, V, generator=gen(V), device="cuda").to(dtype)
            z[0] = inf
            z[1, 5:] = inf
            z[2, 0] = inf
            ids = torch.tensor([1, 2, 0, 3], device="cuda")          # row 2: the token itself is masked
            lp, h, lse = (torch.empty(4, device="cuda") for _ in range(3))
            q.qnn_token_logprobs(z, 4, V, V, ids, lp, entropy=h, lse=lse)
            gl, gh = torch.ones(4, device="cuda"), torch.full((4,), 0.5, device="cuda")
            d = torch.full_like(z, 9.0)
            q.qnn_token_logprobs_backward(z, 4, V, V, ids, lse, h, gl, gh, d, V)
            assert (d[0] == 0).all() and (d[1, 5:] == 0).all() and d[2, 0] == 0 and d.isfinite().all()
            p = (z[1, :5].double() - lse[1].double()).exp()
            logp = z[1, :5].double() - lse[1].double()
            want = -p * (1 + 0.5 * (logp + h[1].double()))
            want[2] += 1
            full = torch.empty(4, V, device="cuda")
            q.qnn_token_logprobs_backward(z.float(), 4, V, V, ids, lse, h, gl, gh, full, V)
            assert ((full[1, :5].double() - want).abs() <= 1e-5).all()
            assert torch.equal(d, full.to(dtype))
            x = z.clone()
            q.qnn_token_logprobs_backward(x, 4, V, V, ids, lse, h, gl, gh, x, V)
            assert torch.equal(x, d)


# ---- streams, graphs, repetition ---------------------------------------------------------------------------------

def test_side_stream_and_graph(q):
    """The calls on another stream than the inputs', captured in a graph and replayed on new inputs, bit for bit."""
    M, K, N, V = 48, 512, 768, 5000
    g = gen(9)
    x = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    r = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    w = torch.randn(N, K, generator=g, device="cuda")
    head = torch.randn(V, N // 2, generator=g, device="cuda")
    cw, sw = torch.empty(N, K, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    ch, sh = torch.empty(V, N // 2, dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    q.qnn_quantize_rows_i8(w, N, K, K, cw, K, sw)
    q.qnn_quantize_rows_i8(head, V, N // 2, N // 2, ch, N // 2, sh)
    ids = torch.randint(0, V, (M,), generator=g, device="cuda")
    s = r.clone()
    c1, s1 = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    c2, s2 = torch.empty(M, N // 2, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    z = torch.empty(M, V, device="cuda")
    lp, h, lse = (torch.empty(M, device="cuda") for _ in range(3))
    tl, ti = torch.empty(M, 5, device="cuda"), torch.empty(M, 5, dtype=torch.int64, device="cuda")
    d = torch.empty_like(z)
    ones = torch.ones(M, device="cuda")

    def chain():
        q.qnn_rmsnorm_quant_i8(x, s, M, K, K, K, None, 1e-5, c1, K, s1, sum_out=s, ld_sum=K)
        q.qnn_gemm_i8_scaled(c1, K, s1, cw, K, sw, M, N, K, y, N)
        q.qnn_silu_mul_quant_i8(y, y[:, N // 2:], M, N // 2, N, N, c2, N // 2, s2)
        q.qnn_gemm_i8_scaled(c2, N // 2, s2, ch, N // 2, sh, M, V, N // 2, z, V)
        q.qnn_token_logprobs(z, M, V, V, ids, lp, entropy=h, lse=lse, topk=5, top_logprob=tl, top_ids=ti)
        q.qnn_token_logprobs_backward(z, M, V, V, ids, lse, h, ones, None, d, V)
    outs = (s, y, z, lp, h, lse, tl, ti, d)
    chain()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    for k in range(3):
        s.copy_(r)
        for o in outs[1:]:
            o.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            chain()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k
    s.copy_(r)
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        chain()
    for k in range(3):
        s.copy_(r)
        for o in outs[1:]:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k
    assert q.qnn_device_status() == 0


def test_every_call_is_one_launch(q):
    """One kernel a call, counted by the library that both the ctypes and the CPython entry share."""
    M, K, N, V = 5, 200, 300, 1000
    x = torch.randn(M, K, device="cuda")
    w = torch.randn(N, K, device="cuda")
    codes, wc = torch.empty(M, 224, dtype=torch.int8, device="cuda"), torch.empty(N, 224, dtype=torch.int8, device="cuda")
    s, ws = torch.empty(M, device="cuda"), torch.empty(N, device="cuda")
    out, z = torch.empty(M, N, device="cuda"), torch.randn(M, V, device="cuda")
    ids = torch.randint(0, V, (M,), device="cuda")
    lp, h, lse = (torch.empty(M, device="cuda") for _ in range(3))
    calls = [lambda: q.qnn_quantize_rows_i8(w, N, K, K, wc, 224, ws),
             lambda: q.qnn_rmsnorm_quant_i8(x, None, M, K, K, K, None, 1e-5, codes, 224, s),
             lambda: q.qnn_silu_mul_quant_i8(x, x, M, K, K, K, codes, 224, s),
             lambda: q.qnn_gemm_i8_scaled(codes, 224, s, wc, 224, ws, M, N, K, out, N),
             lambda: q.qnn_token_logprobs(z, M, V, V, ids, lp, entropy=h, lse=lse),
             lambda: q.qnn_token_logprobs_backward(z, M, V, V, ids, lse, h, lp, h, z, V)]
    for call in calls:
        before = q.qnn_launch_count()
        call()
        assert q.qnn_launch_count() == before + 1
    torch.cuda.synchronize()
    assert q.qnn_device_status() == 0


@pytest.mark.parametrize("M", [1, 2, 4, 9, 16, 40, 130, 600])
def test_product_repeats_bit_for_bit(q, M):
    """The same call again and again gives the same bits, also where K is cut among CTAs or warps."""
    g = gen(M)
    a = torch.randint(-128, 128, (M, 4096), generator=g, device="cuda", dtype=torch.int8)
    b = torch.randint(-128, 128, (520, 4096), generator=g, device="cuda", dtype=torch.int8)
    sa, sb = torch.rand(M, generator=g, device="cuda"), torch.rand(520, generator=g, device="cuda")
    outs = [torch.empty(M, 520, dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    for o in outs:
        q.qnn_gemm_i8_scaled(a, 4096, sa, b, 4096, sb, M, 520, 4096, o, 520)
    assert all(torch.equal(o, outs[0]) for o in outs)


@pytest.mark.parametrize("T,V", [(1, 128000), (6, 90001), (40, 30000), (2000, 3000)])
def test_scores_repeat_bit_for_bit(q, T, V):
    """Rows shared by several CTAs, candidates found in any order: the same numbers and alternatives every time."""
    z = (torch.randn(T, V, generator=gen(T), device="cuda") * 3).bfloat16()
    ids = torch.randint(0, V, (T,), generator=gen(V), device="cuda")
    first = run_scores(q, z, ids, 10, V)
    for _ in range(6):
        assert all(torch.equal(a, b) for a, b in zip(run_scores(q, z, ids, 10, V), first))


# ---- rounding of the codes -----------------------------------------------------------------------------------------

def codes_by_definition(t):
    """round_half_even(t * (127 / max|t|)) in fp32, and max|t| / 127 (numpy: every operation rounded once)."""
    top = np.abs(t).max(1, keepdims=True)
    return np.rint(t * (np.float32(127.0) / top)).astype(np.int8), (top / np.float32(127.0))[:, 0]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", [(400, 16), (300, 512), (64, 1031), (40, 4098), (9, 16400), (5, 20001)])
def test_codes_are_the_definition_bit_for_bit(q, rows, K, dtype):
    """Rows full of ties (t = max * n / 254 with n odd, as nearly as the type holds it): the product is rounded to fp32, then to
    a whole number, in every kernel that quantises; no tolerance."""
    g = gen(rows + K)
    top = torch.rand(rows, 1, generator=g, device="cuda") + 0.5
    n = torch.randint(-127, 127, (rows, K), generator=g, device="cuda") * 2 + 1
    x = (top * n / 254).to(dtype)
    x[:, ::3] = (top * 0.5).to(dtype)                    # 63.5 exactly
    x[:, 1] = top[:, 0].to(dtype)
    o = Quantised(rows, K)
    q.qnn_quantize_rows_i8(x, rows, K, K, o.codes.t, o.ldq, o.scale.t)
    codes, scale = codes_by_definition(x.float().cpu().numpy())
    assert np.array_equal(o.codes.t[:, :K].cpu().numpy(), codes)
    assert np.array_equal(o.scale.t.cpu().numpy(), scale)
    # the norm: u = (x + r) gamma rounds twice more, its factor 1 / rms cancels
    r = torch.randn(rows, K, generator=g, device="cuda").to(dtype) if K % 2 else None
    gamma = torch.exp2(torch.randint(-2, 3, (K,), generator=g, device="cuda").float()).to(dtype) if K % 3 else None
    o = Quantised(rows, K)
    q.qnn_rmsnorm_quant_i8(x, r, rows, K, K, K, gamma, 1e-5, o.codes.t, o.ldq, o.scale.t)
    u = x.float().cpu().numpy()
    u = u + r.float().cpu().numpy() if r is not None else u
    u = u * gamma.float().cpu().numpy() if gamma is not None else u
    assert np.array_equal(o.codes.t[:, :K].cpu().numpy(), codes_by_definition(u)[0])


# ---- waits that run out ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("which", ["QNN_SELFTEST_PRODUCT", "QNN_SELFTEST_SCORES"])
def test_receivers_that_give_up_stay_for_late_senders(q, which):
    """A block of a cluster sends nothing and another late, so that the receivers' waits run out: they report it, are still there
    when the late block's stores arrive, and every later call is as right as before."""
    scratch = torch.empty(q.QNN_SELFTEST_CLUSTER_BYTES, dtype=torch.uint8, device="cuda")
    assert q.qnn_device_status() == 0
    for _ in range(3):
        q.qnn_selftest_cluster_timeout(getattr(q, which), scratch)
        assert q.qnn_device_status() == q.QNN_ERR_TIMEOUT
        assert "wait" in q.qnn_last_error()
        assert q.qnn_device_status() == 0
    check_product(q, 16, 300, 4096, torch.float32)
    z = (torch.randn(3, 20001, generator=gen(8), device="cuda") * 3).bfloat16()
    check_scores(q, z, torch.tensor([5, 0, 20000], device="cuda"), 8, 20001)
    assert q.qnn_device_status() == 0


# ---- norms of tiny rows ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,K", [(9, 1), (9, 96), (40, 200), (9, 1031), (700, 4096), (9, 4097), (9, 16386), (9, 40000)])
def test_rmsnorm_of_rows_whose_squares_underflow(q, rows, K, dtype):
    """eps = 0, or as small as the squares: the sum of squares is below what fp32 holds, the norm is as usual.  1 / rms of a
    64-bit sum rounds once; max / 127 and the product twice more, so scales within 4 U of the exact ones (elsewhere 2e-5)."""
    g = gen(rows + K)
    size = torch.tensor([1e-30, 3e-25, 1e-22, 2e-21, 3e-20, 1e-17, 1e-15, 1.0, 1e-33], device="cuda").repeat(rows // 9 + 1)[:rows]
    x0 = torch.randn(rows, K, generator=g, device="cuda")
    x0[:, 0] = 1.0
    x0 = (x0 * size[:, None]).to(dtype)
    r0 = (torch.randn(rows, K, generator=g, device="cuda") * size[:, None]).to(dtype)
    gamma = (1 + 0.3 * torch.randn(K, generator=g, device="cuda")).to(dtype)
    for eps in (0.0, 1e-40, 1e-30):
        for over in (None, "apart", "x", "residual"):
            x, r = x0.clone(), r0.clone() if over else None
            s64 = x0.float() + r0.float() if over else x0.float()
            want_sum = s64.to(dtype)
            s64 = s64.double()
            t64 = s64 * gamma.double() / torch.sqrt((s64 * s64).mean(1, keepdim=True) + float(np.float32(eps)))
            into = {None: None, "apart": torch.empty_like(x), "x": x, "residual": r}[over]
            o = Quantised(rows, K, values=torch.float32)
            q.qnn_rmsnorm_quant_i8(x, r, rows, K, K, K, gamma, eps, o.codes.t, o.ldq, o.scale.t, sum_out=into, ld_sum=K,
                                   values=o.values.t, ld_values=K)
            if into is not None:
                assert torch.equal(into, want_sum)
            assert o.scale.t.isfinite().all() and o.values.t.isfinite().all()
            # (one element with a residual may come close to nothing: rows below 2^-118 count as zero)
            some = (s64 * gamma.double()).abs().amax(1) > 2.0 ** -117
            top = t64.abs().amax(1)[some] / 127
            assert ((o.scale.t.double()[some] - top).abs() <= 2e-5 * top).all()
            tiny = (s64 * s64).mean(1)[some] + eps < 2.0 ** -98
            assert ((o.scale.t.double()[some] - top).abs()[tiny] <= 4 * U * top[tiny]).all()
            off = o.codes.t[:, :K].double()[some] - t64[some] / top[:, None]
            assert off.abs().max().item() <= 0.5 + 3e-3


# ---- gates far below zero ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [1, 96, 1030, 1031, 4096, 16386, 20001])
def test_silu_down_to_the_end_of_exp(q, K, dtype):
    """Gates of -80 to -88.7, where 1 + exp(-gate) reaches the end of fp32, with factors that keep the product in range; tolerances
    as everywhere (exp is off by (|gate| + 8) U).  Below -88.72 exp overflows, and the gate is 0 whatever it multiplies."""
    big = min(torch.finfo(dtype).max / 8, 1e34)
    gate = torch.empty(6, K, device="cuda")
    for r, (lo, hi) in enumerate([(-88.5, -80.0), (-88.5, -87.0), (-88.0, -88.0), (-87.5, -86.9), (-200.0, -89.0), (-40.0, 3.0)]):
        gate[r] = torch.linspace(hi, lo, K, device="cuda")
    gate = gate.to(dtype)
    up = (torch.rand(6, K, generator=gen(K), device="cuda") * 0.5 + 0.5).to(dtype)
    up[:5] = (up[:5].float() * big).to(dtype)
    o = Quantised(6, K, values=torch.float32)
    q.qnn_silu_mul_quant_i8(gate, up, 6, K, K, K, o.codes.t, o.ldq, o.scale.t, values=o.values.t, ld_values=K)
    assert o.scale.t[4].item() == 0.0 and (o.codes.t[4, :K] == 0).all() and (o.values.t[4] == 0).all()
    a = gate.double()
    t64 = a / (1 + torch.exp(-a)) * up.double()
    top = t64.abs().amax(1)
    for r in (0, 1, 2, 3, 5):
        assert abs(o.scale.t[r].item() * 127 / top[r].item() - 1) < 2e-5, r
        assert (o.codes.t[r, :K].double() - t64[r] * 127 / top[r]).abs().max().item() <= 0.5 + 3e-3, r


# ---- every kernel instance -----------------------------------------------------------------------------------------------------

# odd remainders of tiles, of K blocks and of the shares of K
INSTANCES = [(1, 301, 700), (1, 301, 4001), (2, 1030, 333), (3, 30, 1044), (3, 1728, 4416), (4, 143, 12138),
             (8, 112, 20), (3, 113, 426), (5, 2058, 1060), (6, 489, 2288),
             (30, 2694, 30), (19, 9673, 2880), (19, 295, 1353), (27, 99, 1985),
             (47, 14336, 1366), (41, 10112, 5760), (48, 11008, 2048), (45, 389, 1307), (64, 4096, 4096), (43, 102, 2361),
             (109, 15538, 4352), (100, 16384, 4096), (160, 3392, 14144), (65, 4245, 5562), (90, 2684, 2520), (107, 153, 5154),
             (169, 75, 41), (65, 745, 245), (46, 9502, 630), (524, 3149, 1129), (900, 1856, 2752), (133, 4738, 2528),
             (153, 10338, 682), (1846, 1431, 1315), (701, 4096, 4096), (1442, 2465, 1947), (134, 16473, 1322), (10000, 4096, 4096)]


def test_instances_are_all_of_them(q):
    """The products below run on every kernel that the choice by cost can reach, with rows that leave as bulk stores or 16-byte
    stores, and with rows that leave element by element."""
    every = {(q.QNN_I8S_TOKENS, c, r) for c, r in ((1, 4), (1, 2), (2, 4), (4, 4))}
    every |= {(q.QNN_I8S_NARROW, c, s) for c in (16, 32, 64, 128) for s in (1, 2, 4, 8)}
    every |= {(q.QNN_I8S_WIDE, c, s) for c, s in ((64, 1), (128, 1), (128, 2), (192, 2), (256, 2))}
    for round_to in (lambda N: N // 8 * 8, lambda N: N | 1):
        reached = {q.qnn_gemm_i8_scaled_kernel(M, round_to(N), K) for M, N, K in INSTANCES}
        assert reached == every, (every - reached, reached - every)
    assert q.qnn_gemm_i8_scaled_kernel(5, 5, 0) == q.qnn_gemm_i8_scaled_kernel(0, 5, 5) == (0, 0, 0)


@pytest.mark.parametrize("M,N,K", INSTANCES)
def test_product_instances(q, M, N, K):
    for n, dtypes in ((N // 8 * 8, TYPES), (N | 1, TYPES[:2])):
        for dtype in dtypes:
            check_product(q, M, n, K, dtype, bias=dtype != torch.float16, seed=1)
    assert q.qnn_device_status() == 0


# ---- scores: nothing lost, nothing counted twice --------------------------------------------------------------------------------

LONG_SCORES = [(5, 40), (130, 1000), (2000, 2560), (300, 5003), (1100, 8001), (700, 16384), (64, 32000), (33, 50021), (200, 65536), (1, 70001),
               (4, 128001), (40, 128000), (3, 300001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", LONG_SCORES)
def test_scores_count_every_logit(q, T, V, dtype):
    """Equal logits: every e^(z - m) is 1 and the sum is the whole number V, exactly, in any order; what is left is one logarithm
    (2 units of its value) and one rounding.  A logit more or less moves it by 1 / V, 30 times that at V = 300001."""
    for value, ld, off in ((0.0, V, 0), (1.5, V + 3, 1)):
        z = torch.full((off + T * ld,), float("nan"), dtype=dtype, device="cuda")[off:].view(T, ld)[:, :V]
        z.fill_(value)
        ids = torch.randint(0, V, (T,), generator=gen(V), device="cuda")
        lp, h, lse, _, _ = run_scores(q, z, ids, 0, ld)
        log = float(np.log(np.float64(V)))
        assert ((lse.double() - (value + log)).abs() <= 4 * U * (value + log)).all()
        assert ((h.double() - log).abs() <= 4 * U * log).all()
        assert ((lp.double() + log).abs() <= 4 * U * log).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(40, 40), (1031, 1031), (5003, 5003), (600, 50021), (5, 131077), (3, 300001), (64, 131077)])
def test_scores_find_every_place(q, T, V, dtype):
    """One logit left among masked ones, in another place in every row (in every place, where there are as many rows): e^0 is the
    whole sum, so every number is exact, and it is the best alternative."""
    g = gen(T + V)
    at = torch.arange(T, device="cuda") if T == V else torch.randint(0, V, (T,), generator=g, device="cuda")
    if T < V:                                            # the ends, and both sides of where a row is cut in two, four or eight
        edges = [0, V - 1, V // 2, V // 2 + 7, V // 8, V // 4 - 1, V - 9]
        at[:min(T, 7)] = torch.tensor(edges[:min(T, 7)], device="cuda")
    for value in (0.0, -7.5):
        z = torch.full((T, V), float("-inf"), device="cuda", dtype=dtype)
        z.scatter_(1, at[:, None], value)
        lp, h, lse, tl, ti = run_scores(q, z, at, 1, V)
        assert (lse == value).all() and (lp == 0).all() and (h == 0).all() and (tl == 0).all()
        assert torch.equal(ti[:, 0], at)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", LONG_SCORES)
def test_scores_of_rising_and_falling_rows(q, T, V, dtype):
    """Rows that rise, so that the running maximum moves in every step and all that was added is rescaled (by a factor off by
    8 units), rows that fall, and rows that are mostly low with a high end.  A thread adds at most V / (2 * threads) terms in
    turn, exp is off by (3 |z - m| + 4) units and counts by its probability."""
    ramp = torch.linspace(-3.0, 0.0, V, device="cuda")
    late = torch.where(torch.arange(V, device="cuda") >= V - max(1, V // 50), 0.0, -2.0)
    z = torch.stack([(ramp, ramp.flip(0), late, late.flip(0))[t % 4] for t in range(min(T, 8))]).to(dtype)
    z = z.repeat((T + z.shape[0] - 1) // z.shape[0], 1)[:T].contiguous()
    ids = torch.randint(0, V, (T,), generator=gen(V), device="cuda")
    lp, h, lse, _, _ = run_scores(q, z, ids, 0, V)
    z64 = z.double()
    logp = torch.log_softmax(z64, 1)
    h64 = -(logp.exp() * logp).sum(1)
    lse64 = torch.logsumexp(z64, 1)
    threads = 64 if V <= 8192 else 128 if V <= 65536 else 256
    steps = V / (threads * (16 if dtype == torch.float32 else 32))      # rounds, and so rescales
    tol = U * (V / (2 * threads) + 8 * steps + 24 + 13 + 3 * lse64)
    assert ((lse.double() - lse64).abs() <= tol).all()
    assert ((lp.double() - logp.gather(1, ids[:, None])[:, 0]).abs() <= tol + 3 * U).all()
    assert ((h.double() - h64).abs() <= tol * (1 + 2 * 3.0) + 3 * U * h64).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(500, 2000), (200, 32000), (100, 128000)])
def test_scores_errors_are_roundings(q, T, V, dtype):
    """Over many rows of random logits: the errors of hundreds of partial sums average out, so the root mean square is that of the
    last operations -- a logarithm, a sum, exp's own bias -- and not of the terms' number."""
    z = (torch.randn(T, V, generator=gen(T), device="cuda") * 3).to(dtype)
    ids = torch.randint(0, V, (T,), generator=gen(V), device="cuda")
    lp, h, lse, _, _ = run_scores(q, z, ids, 0, V)
    logp = torch.log_softmax(z.double(), 1)
    lse64, h64 = torch.logsumexp(z.double(), 1), -(logp.exp() * logp).sum(1)

    def rms(x):
        return x.square().mean().sqrt().item()
    assert rms(lse.double() - lse64) <= U * (lse64.mean().item() + 8)
    assert rms(lp.double() - logp.gather(1, ids[:, None])[:, 0]) <= U * (-lp.double().mean().item() + 2 * lse64.mean().item() + 8)
    assert rms(h.double() - h64) <= U * (2 * h64.mean().item() + 2 * lse64.mean().item() + 16)


# ---- gradients of batches long enough for several rounds a block ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES[1:])
@pytest.mark.parametrize("T,V", [(400, 60001), (600, 60001), (1000, 60001), (300, 262147)])
def test_scores_gradient_of_long_batches(q, T, V, dtype):
    """16-bit batches of 20 to 80 million logits (two to four rounds a block), a token in every round: the fp32 gradient rounded
    once, bit for bit, and that within its tolerance of 64 bits."""
    g = gen(T + V)
    z = (torch.randn(T, V, generator=g, device="cuda") * 2.5).to(dtype)
    ids = (torch.arange(T, device="cuda") * (V // T) + torch.randint(0, V // T, (T,), generator=g, device="cuda"))
    lp, h, lse = (torch.empty(T, device="cuda") for _ in range(3))
    q.qnn_token_logprobs(z, T, V, V, ids, lp, entropy=h, lse=lse)
    gl, gh = torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda") * 0.1
    d = Guarded((T, V), dtype)
    q.qnn_token_logprobs_backward(z, T, V, V, ids, lse, h, gl, gh, d.t, V)
    d.check()
    full = torch.empty(T, V, device="cuda")
    zf = z.float()
    q.qnn_token_logprobs_backward(zf, T, V, V, ids, lse, h, gl, gh, full, V)
    assert torch.equal(d.t, full.to(dtype))
    for rows in range(0, T, 100):
        s = slice(rows, rows + 100)
        x = zf[s].double() - lse[s].double()[:, None]
        p = x.exp()
        want = -p * (gl[s].double()[:, None] + gh[s].double()[:, None] * (x + h[s].double()[:, None]))
        want.scatter_add_(1, ids[s][:, None], gl[s].double()[:, None])
        # exp is off by (3 |x| + 4) units, the factor by 3 of its terms, the token's sum by one of its own
        terms = p * (gl[s].double().abs()[:, None] + gh[s].double().abs()[:, None] * (x.abs() + h[s].double()[:, None]))
        tol = U * terms * (3 * x.abs() + 10) + 2 * U * want.abs() + 1e-37
        assert ((full[s].double() - want).abs() <= tol).all()


# ---- scales ------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", [(1, 4096), (3, 1), (400, 1000), (33, 4097), (700, 4096), (5, 11010), (5, 16386), (3, 20001), (9, 33000)])
def test_scales_of_norm_and_gate(q, rows, K, dtype):
    """The norm: a thread adds at most K / 1024 + 32 squares in turn and a tree 12 sums, of which the root halves the error; s * gamma,
    max / 127, the root, its reciprocal and the product round once each (the root and the reciprocal within two units).  The gate:
    exp within (3 |a| + 4) units, the reciprocal within 2, three products, one division."""
    g = gen(rows + K)
    x, r = ((torch.randn(rows, K, generator=g, device="cuda") * 2).to(dtype) for _ in range(2))
    gamma = (1 + 0.3 * torch.randn(K, generator=g, device="cuda")).to(dtype)
    o = Quantised(rows, K)
    q.qnn_rmsnorm_quant_i8(x, r, rows, K, K, K, gamma, 1e-6, o.codes.t, o.ldq, o.scale.t)
    s64 = (x.float() + r.float()).double()
    want = (s64 * gamma.double()).abs().amax(1) / 127 / torch.sqrt((s64 * s64).mean(1) + float(np.float32(1e-6)))
    assert ((o.scale.t.double() - want).abs() <= U * ((K / 1024 + 32 + 12) / 2 + 8) * want).all()
    o = Quantised(rows, K)
    q.qnn_silu_mul_quant_i8(x, r, rows, K, K, K, o.codes.t, o.ldq, o.scale.t)
    a = x.double()
    want = (a / (1 + torch.exp(-a)) * r.double()).abs().amax(1) / 127
    assert ((o.scale.t.double() - want).abs() <= U * (3 * a.abs().amax(1) + 4 + 2 + 4) * want).all()


# ---- scores while other rows keep the SM busy ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,topk", [(232, 171761, 32), (453, 88169, 32), (710, 56298, 32), (345, 115791, 20), (1500, 9001, 32), (30, 300001, 32)])
def test_scores_stand_beside_rows_that_look_for_alternatives(q, T, V, topk, dtype):
    """Rows stream while others on the same SM read theirs again for many alternatives: whatever that does to the timing of their
    copies, every call gives the same bits, and those within the roundings of random rows."""
    ld = V + 3
    z = strided(T, V, ld, dtype, 1, gen(T + V), 3.0)
    ids = torch.randint(0, V, (T,), generator=gen(V), device="cuda")
    check_scores(q, z, ids, topk, ld)
    first = run_scores(q, z, ids, topk, ld)
    lse64 = torch.logsumexp(z.double(), 1)
    assert (first[2].double() - lse64).abs().max().item() <= 40 * U * (1 + lse64.max().item())
    for _ in range(30):
        assert all(torch.equal(a, b) for a, b in zip(run_scores(q, z, ids, topk, ld), first))
