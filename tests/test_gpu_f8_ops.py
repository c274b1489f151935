"""The calls on 8-bit floating point with block scales against plain formulas in 64 bits.

Tolerances.  Scales and codes are exact: the scale is read off the largest magnitude, and a code is one rounding of an exact
quotient, so both are compared bit for bit with the nearest number of the type, found in 64 bits.  A product of two codes is
exact; sums are held in fp32.  Where all partial sums are multiples of one unit and below 2^24 of it, every order of adding gives the
same number, and results are compared bit for bit: most product tests are made so.  In general each of the K terms may lose up to a
unit in the last place (2^-23) of the sum of magnitudes S, whatever the order: K 2^-23 S.  16-bit results are the fp32 results of the
same call rounded once, bit for bit.
"""
import pytest
import torch

from util import Guarded

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
CODES = {torch.float8_e4m3fn: (8, 448.0, -6, 3), torch.float8_e5m2: (15, 57344.0, -14, 2)}
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
B = 128


@pytest.fixture(scope="module")
def q():
    import paper_1609_07061_b200.binding as b
    yield b
    assert b.qnn_device_status() == 0


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def up(n, to):
    return (n + to - 1) // to * to


# ---- the format in 64 bits -----------------------------------------------------------------------------------------

def ref_scale(top, code):
    """Scale bytes of blocks with these largest magnitudes (double)."""
    x, most, _, _ = CODES[code]
    e = torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / most))
    e = torch.where(torch.exp2(e) * most < top, e + 1, torch.where(torch.exp2(e - 1) * most >= top, e - 1, e))
    s = (e.clamp(min=-127) + 127)
    s = torch.where(top > 0, s, torch.zeros_like(s))
    return torch.where(torch.isfinite(top), s, torch.full_like(s, 255)).to(torch.uint8)


def ref_round(v, code):
    """Nearest number of the type (double), ties to even; v within its range."""
    _, _, low, bits = CODES[code]
    ulp = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** low))) - bits)
    return (v / ulp).round() * ulp


def ref_blocks(x, rows, cols, code):
    """[R, C] double -> the values that codes stand for divided by their scale, and scale bytes, in blocks of rows x cols."""
    R, C = x.shape
    p = torch.nn.functional.pad(x, (0, up(C, cols) - C, 0, up(R, rows) - R))
    b = p.view(p.shape[0] // rows, rows, p.shape[1] // cols, cols)
    top = b.abs().amax(3).amax(1)
    top = torch.where(b.isnan().any(3).any(1), torch.full_like(top, float("inf")), top)
    s = ref_scale(top, code)
    bad = (s == 255)[:, None, :, None]
    v = torch.where(bad, torch.zeros_like(b), b * torch.exp2(127.0 - s.double())[:, None, :, None])
    return ref_round(v, code).reshape(p.shape)[:R, :C], s


def expand(s, rows, cols, R, C):
    """Factors of scale bytes, one an element (NaN for 255)."""
    f = torch.exp2(s.double() - 127)
    f = torch.where(s == 255, torch.full_like(f, float("nan")), f)
    return f.repeat_interleave(rows, 0)[:R].repeat_interleave(cols, 1)[:, :C]


def strided(rows, K, ld, dtype, offset, g, scale=1.0):
    """[rows, K] view with row stride ld, `offset` elements into its buffer; the rest of the buffer is NaN."""
    buf = torch.full((offset + rows * ld + 16,), float("nan"), dtype=dtype, device="cuda")
    v = buf[offset:offset + rows * ld].view(rows, ld)[:, :K]
    v.copy_((torch.randn(rows, K, generator=g, device="cuda") * scale * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).to(dtype))
    return v


class Out:
    """Guarded codes, scales and values of a quantising call."""

    def __init__(self, rows, K, scale_rows, scale_cols, code, values=None, ldq=None, ldv=None):
        self.rows, self.K, self.code = rows, K, code
        self.ldq, self.lds, self.ldv = ldq or up(K, 16) + 16, up(scale_cols, 16) + 16, ldv or K
        self.codes, self.scale = Guarded((rows, self.ldq), torch.uint8), Guarded((scale_rows, self.lds), torch.uint8)
        self.values = Guarded((rows, self.ldv), values) if values else None
        self.q = self.codes.t.view(code)

    def check(self, want, s, block, rows=None):
        """want: codes (double), s: scale bytes; rows: how many are written."""
        rows = self.rows if rows is None else rows
        for b in (self.codes, self.scale, self.values):
            if b is not None:
                b.check()
        assert torch.equal(self.scale.t[:s.shape[0], :s.shape[1]], s)
        assert torch.equal(self.q[:rows, :self.K].double(), want)
        K16 = up(self.K, 16)
        assert (self.codes.t[:rows, self.K:K16] == 0).all(), "codes up to the next 16 are zero"
        assert (self.codes.t[:rows, K16:] == 0xA5).all(), "bytes past them are untouched"
        assert (self.codes.t[rows:] == 0xA5).all() and (self.scale.t[s.shape[0]:] == 0xA5).all(), "rows behind are untouched"
        if self.values is not None:
            v = (want * expand(s, *block, rows, self.K)).to(torch.float32).to(self.values.dtype)
            got = self.values.t[:rows, :self.K]
            assert torch.equal(got.isnan(), v.isnan()) and torch.equal(got.nan_to_num(0.0), v.nan_to_num(0.0))


SHAPES = [(1, 1), (3, 7), (2, 16), (5, 100), (1, 128), (9, 129), (7, 255), (3, 256), (130, 1000), (2, 1025), (1, 4096), (3, 4097), (301, 640),
          (33, 2050), (128, 136), (129, 8192), (2, 16385)]


def layouts(K):
    # dense; padded and aligned; rows of even offset; rows of odd offset
    return enumerate([(K, 0), (up(K, 8) + 8, 0), (up(K, 2), 2), (K + 3, 1)])


@pytest.mark.parametrize("code", [E4M3, E5M2])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", SHAPES)
def test_quantize_blocks(q, rows, K, dtype, code):
    g = gen(rows * 7 + K)
    for n, (ld, off) in layouts(K):
        x = strided(rows, K, ld, dtype, off, g, 3.0)
        o = Out(rows, K, rows, up(K, B) // B, code, TYPES[n % 3], ldv=K + (n % 2))
        q.qnn_quantize_blocks_f8(x, rows, K, ld, o.q, o.ldq, o.scale.t, o.lds, values=o.values.t, ld_values=o.ldv)
        o.check(*ref_blocks(x.double(), 1, B, code), (1, B))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_blocks_by_index(q, dtype):
    for rows, src, K in [(1, 5, 100), (40, 7, 1000), (300, 64, 2048), (17, 3, 129)]:
        g = gen(rows)
        x = strided(src, K, K + 1, dtype, 0, g)
        index = torch.randint(0, src, (rows,), generator=g, device="cuda")
        index[rows // 2] = -1                                   # rows that are not there
        index[rows // 3] = src
        if rows > 2:
            index[-1] = 2 ** 40
        there = (index >= 0) & (index < src)
        want = torch.where(there[:, None], x[index.clamp(0, src - 1)].double(), torch.zeros(1, device="cuda", dtype=torch.float64))
        o = Out(rows, K, rows, up(K, B) // B, E4M3, torch.bfloat16)
        q.qnn_quantize_blocks_f8(x, rows, K, K + 1, o.q, o.ldq, o.scale.t.view(torch.float8_e8m0fnu), o.lds, index=index, src_rows=src,
                                 values=o.values.t, ld_values=o.ldv)
        o.check(*ref_blocks(want, 1, B, E4M3), (1, B))


@pytest.mark.parametrize("code", [E4M3, E5M2])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", SHAPES)
def test_quantize_tiles(q, rows, K, dtype, code):
    g = gen(rows * 11 + K)
    for n, (ld, off) in layouts(K):
        x = strided(rows, K, ld, dtype, off, g, 3.0)
        o = Out(rows, K, up(rows, B) // B, up(K, B) // B, code, TYPES[n % 3], ldv=K + (n % 2))
        q.qnn_quantize_tiles_f8(x, rows, K, ld, o.q, o.ldq, o.scale.t, o.lds, values=o.values.t, ld_values=o.ldv)
        o.check(*ref_blocks(x.double(), B, B, code), (B, B))


GROUPS = [[5], [0], [128], [129, 0, 1], [0, 0, 300, 0], [37] * 40, [1] * 33 + [500] + [0] * 33 + [2]]


def padded(x, sizes, first=0):
    out = torch.zeros(sum(up(n, B) for n in sizes), x.shape[1], dtype=x.dtype, device=x.device)
    at, to = first, 0
    for n in sizes:
        out[to:to + n] = x[at:at + n]
        at, to = at + n, to + up(n, B)
    return out


def offsets_of(sizes, first=0):
    return (torch.tensor([0] + list(sizes), dtype=torch.int64).cumsum(0) + first).cuda()


@pytest.mark.parametrize("code", [E4M3, E5M2])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", GROUPS, ids=lambda s: f"{len(s)}x{sum(s)}")
def test_quantize_columns(q, sizes, dtype, code):
    for n, (K, first, behind) in enumerate([(100, 0, 0), (136, 3, 5), (1, 0, 1), (1025, 2, 0)]):
        g = gen(len(sizes) + K)
        M, G = first + sum(sizes) + behind, len(sizes)
        ld = K + n
        x = strided(max(M, 1), K, ld, dtype, n, g)
        blocks = M // B + G
        o = Out(blocks * B, K, blocks, K, code, TYPES[n % 3])
        q.qnn_quantize_columns_f8(x, M, K, ld, offsets_of(sizes, first), G, o.q, o.ldq, o.scale.t, o.lds, values=o.values.t, ld_values=o.ldv)
        want, s = ref_blocks(padded(x.double(), sizes, first), B, 1, code)
        o.check(want, s, (B, 1), rows=want.shape[0])


def test_quantisers_at_the_ends_of_the_range(q):
    """Zeros, subnormals, the border of a scale, the largest numbers, infinities and NaN, each in a block of its own."""
    for code, (x, most, _, _) in CODES.items():
        tiny = 2.0 ** -149
        rows = [[0.0], [-0.0], [tiny], [2.0 ** -126, tiny], [most, 1.0], [most * (1 + 2.0 ** -23), 1.0], [most * 2.0 ** -119], [1e-38, -3e-39],
                [3.4e38, 1.0], [3.4028234663852886e38, -3.4e38], [float("inf"), 1.0], [1.0, float("-inf")], [float("nan"), 2.0], [1.0, -1.0], [most / 2, most / 4],
                [17.0, 19.0, most], [1.0625, 1.1875, 1.3125]]
        t = torch.zeros(len(rows), B, device="cuda")
        for i, r in enumerate(rows):
            t[i, :len(r)] = torch.tensor(r)
        o = Out(len(rows), B, len(rows), 1, code, torch.float32)
        q.qnn_quantize_blocks_f8(t, len(rows), B, B, o.q, o.ldq, o.scale.t, o.lds, values=o.values.t, ld_values=o.ldv)
        o.check(*ref_blocks(t.double(), 1, B, code), (1, B))
        assert o.scale.t[10:13, 0].tolist() == [255] * 3
        # the same as columns and as tiles of a row each
        cols = t.t().contiguous()
        o = Out(2 * B, len(rows), 2, len(rows), code, torch.float32)
        q.qnn_quantize_columns_f8(cols, B, len(rows), len(rows), None, 1, o.q, o.ldq, o.scale.t, o.lds, values=o.values.t, ld_values=o.ldv)
        o.check(*ref_blocks(cols.double(), B, 1, code), (B, 1), rows=B)
        for i in range(len(rows)):
            o = Out(1, B, 1, 1, code, torch.float32)
            q.qnn_quantize_tiles_f8(t[i:i + 1], 1, B, B, o.q, o.ldq, o.scale.t, o.lds, values=o.values.t, ld_values=o.ldv)
            o.check(*ref_blocks(t[i:i + 1].double(), B, B, code), (B, B))


# ---- products ------------------------------------------------------------------------------------------------------

def small_codes(g, rows, cols, code, pad=0):
    """Codes -2, -1, 0, 1, 2 (rows `cols` rounded up to 16 plus pad apart; what stands behind a row is NaN)."""
    ld = up(cols, 16) + pad
    buf = torch.full((rows, ld), 0x7f, dtype=torch.uint8, device="cuda")
    v = torch.randint(-2, 3, (rows, cols), generator=g, device="cuda")
    buf[:, :cols] = v.float().to(code).view(torch.uint8)
    return buf.view(code), v.double()


def small_scales(g, rows, cols, spread=2):
    """Bytes around 127; what stands behind a row is 255."""
    buf = torch.full((rows, up(cols, 16)), 255, dtype=torch.uint8, device="cuda")
    buf[:, :cols] = torch.randint(127 - spread, 128 + spread, (rows, cols), generator=g, device="cuda").to(torch.uint8)
    return buf, buf[:, :cols]


class Operand:
    def __init__(self, g, rows, cols, code, block, pad=0, spread=2):
        self.codes, v = small_codes(g, rows, cols, code, pad)
        self.scale, s = small_scales(g, up(rows, block[0]) // block[0], up(cols, block[1]) // block[1], spread)
        self.ld, self.lds = self.codes.shape[1], self.scale.shape[1]
        self.exact = v * expand(s, *block, rows, cols)


def weights(g, groups, rows, cols, code, pad=0):
    ws = [Operand(g, rows, cols, code, (B, B), pad) for _ in range(groups)]
    codes = torch.stack([w.codes.view(torch.uint8) for w in ws]).view(code)
    return codes, torch.stack([w.scale for w in ws]), ws


def check_out(got, want64, rows=None):
    """Exact sums: fp32 results equal the 64-bit ones, 16-bit results those rounded once."""
    got.check()
    want = want64.to(torch.float32)
    assert (want.double() == want64).all(), "the test's sums are meant to be exact"
    assert torch.equal(got.t[:, :want.shape[1]], want.to(got.dtype))


PRODUCTS = [(1, 1, 1), (1, 128, 128), (2, 40, 100), (3, 130, 129), (16, 256, 512), (17, 300, 640), (33, 128, 2048), (47, 1000, 516), (65, 129, 1000),
            (100, 513, 1111), (128, 384, 128), (129, 260, 300), (240, 128, 256), (241, 1024, 260), (300, 2047, 1111), (500, 384, 4096),
            (1023, 136, 777), (2000, 640, 144)]


@pytest.mark.parametrize("across", [False, True], ids=["forward", "across"])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product_exact(q, M, N, K, across):
    for n, (a_code, b_code, out) in enumerate([(E4M3, E4M3, torch.float32), (E5M2, E4M3, torch.bfloat16), (E4M3, E5M2, torch.float16),
                                               (E5M2, E5M2, torch.float32)]):
        g = gen(M + N + K + n)
        a = Operand(g, M, K, a_code, (1, B), pad=16 * (n % 2))
        w = Operand(g, K if across else N, N if across else K, b_code, (B, B), pad=16 * (n // 2))
        bias = torch.randint(-8, 9, (N,), generator=g, device="cuda").float() if n % 2 else None
        ldo = N + [0, 5, 8, 1][n]
        o = Guarded((M, ldo), out)
        q.qnn_gemm_f8(a.codes, a.ld, a.scale, a.lds, w.codes, w.ld, w.scale, w.lds, M, N, K, o.t, ldo, bias=bias, b_transposed=across)
        want = a.exact @ (w.exact if across else w.exact.t())
        check_out(o, want + bias.double() if bias is not None else want)
        if ldo > N:
            assert (o.t[:, N:].contiguous().view(torch.uint8) == 0xA5).all()


@pytest.mark.parametrize("across", [False, True], ids=["forward", "across"])
@pytest.mark.parametrize("sizes", GROUPS + [[300, 0, 17, 1000, 1], [2000, 3], [64] * 16], ids=lambda s: f"{len(s)}x{sum(s)}")
def test_grouped_exact(q, sizes, across):
    for n, (N, K, first, behind) in enumerate([(128, 128, 0, 0), (300, 516, 3, 2), (129, 100, 0, 40), (640, 1029, 1, 0)]):
        g = gen(sum(sizes) + N + n)
        M, G = first + sum(sizes) + behind, len(sizes)
        if M == 0:
            continue
        a = Operand(g, M, K, E4M3, (1, B))
        codes, scales, ws = weights(g, G, K if across else N, N if across else K, E4M3)
        bias = torch.randint(-8, 9, (G, N), generator=g, device="cuda").float() if n % 2 else None
        o = Guarded((M, N), TYPES[n % 3])
        before = o.t.clone()
        q.qnn_gemm_f8_grouped(a.codes, a.ld, a.scale, a.lds, codes, codes.shape[2], scales, scales.shape[2], offsets_of(sizes, first), G, M, N, K,
                              o.t, N, bias=bias, b_transposed=across)
        o.check()
        at = first
        for i, rows in enumerate(sizes):
            want = a.exact[at:at + rows] @ (ws[i].exact if across else ws[i].exact.t())
            if bias is not None:
                want = want + bias[i].double()
            assert torch.equal(o.t[at:at + rows], want.to(torch.float32).to(o.dtype))
            at += rows
        same = lambda s: torch.equal(o.t[s].view(torch.uint8), before[s].view(torch.uint8))
        assert same(slice(0, first)) and same(slice(at, M)), "rows of no group are left as they were"


@pytest.mark.parametrize("sizes", GROUPS + [[300, 0, 17, 1000, 1], [2000, 3]], ids=lambda s: f"{len(s)}x{sum(s)}")
def test_weight_gradient_exact(q, sizes):
    for n, (N, K) in enumerate([(128, 128), (300, 516), (1, 240), (129, 241), (16, 1), (520, 1029)]):
        g = gen(sum(sizes) + N + n)
        M, G = sum(sizes), len(sizes)
        y_code, x_code = [(E4M3, E4M3), (E5M2, E4M3), (E4M3, E5M2)][n % 3]
        blocks = [up(s, B) // B for s in sizes]
        rows = sum(blocks) * B
        y, x = Operand(g, max(rows, B), N, y_code, (B, 1)), Operand(g, max(rows, B), K, x_code, (B, 1))
        # rows that fill a group up are zeros, as the quantiser writes them
        at = 0
        for s, nb in zip(sizes, blocks):
            for t in (y, x):
                t.codes.view(torch.uint8)[at + s:at + nb * B] = 0
                t.exact[at + s:at + nb * B] = 0
            at += nb * B
        ld = K + [0, 8, 3][n % 3]
        o = Guarded((G * N, ld), TYPES[n % 3])
        q.qnn_gemm_f8_wgrad(y.codes, y.ld, y.scale, y.lds, x.codes, x.ld, x.scale, x.lds, offsets_of(sizes), G, M, N, K, o.t, ld)
        o.check()
        at = 0
        for i, nb in enumerate(blocks):
            want = y.exact[at:at + nb * B].t() @ x.exact[at:at + nb * B]
            assert torch.equal(o.t[i * N:(i + 1) * N, :K], want.to(torch.float32).to(o.dtype)), (i, N, K)
            at += nb * B
        if ld > K:
            assert (o.t[:, K:].contiguous().view(torch.uint8) == 0xA5).all()


def test_tensors_on_another_device_are_refused(q):
    x, c, s = torch.zeros(64, 64, device="cuda"), torch.zeros(64, 64, dtype=torch.uint8, device="cuda").view(E4M3), torch.zeros(64, 16, dtype=torch.uint8, device="cuda")
    i, before = torch.zeros(3, dtype=torch.int64, device="cuda"), q.qnn_launch_count()
    calls = [(lambda x, c, s, i: q.qnn_quantize_blocks_f8(x, 64, 64, 64, c, 64, s, 16, index=i, src_rows=64)),
             (lambda x, c, s, i: q.qnn_quantize_columns_f8(x, 64, 16, 64, i, 2, c, 64, s, 16)),
             (lambda x, c, s, i: q.qnn_gemm_f8_grouped(c, 64, s, 16, c, 64, s, 16, i, 2, 4, 4, 64, x, 4))]
    for f in calls:
        for n in range(4):
            t = [x, c, s, i]
            t[n] = t[n].cpu()
            with pytest.raises(ValueError):
                f(*t)
    for f in (lambda w: q.qnn_quantize_tiles_f8(w, 64, 64, 64, c, 64, s, 16), lambda w: q.qnn_gemm_f8(c, 64, s, 16, c, 64, s, 16, 4, 4, 64, w, 4),
              lambda w: q.qnn_gemm_f8_wgrad(c, 64, s, 16, c, 64, s, 16, i, 2, 64, 16, 16, w, 16)):
        with pytest.raises(ValueError):
            f(x.cpu())
    assert q.qnn_launch_count() == before


@pytest.mark.parametrize("top,other", [(254, 0), (0, 254), (0, 0), (1, 126), (1, 127), (254, 127), (254, 128), (200, 60)])
def test_weight_gradient_scales_at_the_ends(q, top, other):
    """One channel's and one column's scale far from the others: powers of two that are no fp32 numbers by themselves, results exact."""
    g, N, K = gen(top * 256 + other), 130, 140
    y, x = Operand(g, B, N, E4M3, (B, 1), spread=0), Operand(g, B, K, E4M3, (B, 1), spread=0)
    yv, xv = y.codes[:, :N].double(), x.codes[:, :K].double()
    y.scale[0, 7] = top
    x.scale[0, 9] = other
    o = Guarded((N, K), torch.float32)
    q.qnn_gemm_f8_wgrad(y.codes, y.ld, y.scale, y.lds, x.codes, x.ld, x.scale, x.lds, offsets_of([B]), 1, B, N, K, o.t, K)
    o.check()
    f = lambda s, n: torch.exp2(s[0, :n].double() - 127)
    want = (yv.t() @ xv) * f(y.scale, N)[:, None] * f(x.scale, K)[None]
    # a small integer (10 bits) times a power of two: fp32 holds it, but for what is rounded once (below 2^-126) or overflows
    assert torch.equal(o.t, want.float())


def test_weight_gradient_nan_scales_stay_in_their_channel_and_column(q):
    g, sizes, N, K = gen(5), [130, 0, 100], 140, 150
    y, x = Operand(g, 3 * B, N, E4M3, (B, 1)), Operand(g, 3 * B, K, E5M2, (B, 1))
    y.codes.view(torch.uint8)[130:256] = 0
    y.codes.view(torch.uint8)[356:] = 0
    y.scale[1, 3] = 255
    x.scale[2, 139] = 255
    o = Guarded((3 * N, K), torch.float32)
    q.qnn_gemm_f8_wgrad(y.codes, y.ld, y.scale, y.lds, x.codes, x.ld, x.scale, x.lds, offsets_of(sizes), 3, 230, N, K, o.t, K)
    o.check()
    bad = o.t.view(3, N, K).isnan()
    want = torch.zeros_like(bad)
    want[0, 3] = True
    want[2, :, 139] = True
    assert torch.equal(bad, want)


def test_weight_gradient_offsets_that_fall_or_leave_the_rows(q):
    """Held to rise and to stay within 0..M: the same as the offsets they are held to."""
    g, N, K, M = gen(6), 33, 40, 300
    y, x = Operand(g, 8 * B, N, E4M3, (B, 1)), Operand(g, 8 * B, K, E4M3, (B, 1))
    out = []
    for offs in ([-5, 200, 100, 900, 50], [0, 200, 200, 300, 300]):
        o = Guarded((4 * N, K), torch.float32)
        t = torch.tensor(offs, dtype=torch.int64, device="cuda")
        q.qnn_gemm_f8_wgrad(y.codes, y.ld, y.scale, y.lds, x.codes, x.ld, x.scale, x.lds, t, 4, M, N, K, o.t, K)
        o.check()
        out.append(o.t.clone())
    assert torch.equal(*out) and (out[0].view(4, N, K)[[1, 3]] == 0).all() and (out[0].view(4, N, K)[[0, 2]] != 0).any()


def test_weight_gradient_captured_and_on_two_streams(q):
    g, N, K = gen(7), 200, 260
    y, x = Operand(g, 4 * B, N, E4M3, (B, 1)), Operand(g, 4 * B, K, E4M3, (B, 1))
    off = offsets_of([2 * B, 2 * B])
    outs = [torch.zeros(2 * N, K, device="cuda") for _ in range(4)]
    call = lambda o: q.qnn_gemm_f8_wgrad(y.codes, y.ld, y.scale, y.lds, x.codes, x.ld, x.scale, x.lds, off, 2, 4 * B, N, K, o, K)
    call(outs[0])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s, o in zip(streams, outs[1:3]):
        with torch.cuda.stream(s):
            call(o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[3])
    for _ in range(2):
        outs[3].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[0], o) for o in outs[1:]) and (outs[0] != 0).any()


def within(got, a, b, terms):
    """|got - a b| <= terms 2^-23 |a| |b|, and half a step of a 16-bit result."""
    want, s = a @ b, a.abs() @ b.abs()
    eps = torch.finfo(got.dtype).eps / 2
    slack = terms * 2.0 ** -23 * s * (1 + eps) + (eps * want.abs() if got.dtype != torch.float32 else 0)
    assert ((got.double() - want).abs() <= slack + 2.0 ** -149).all()


def quantised(call, rows, K, scale_rows, scale_cols, code):
    """(codes, scale bytes, what they stand for) of a quantising call."""
    c = torch.zeros(rows, up(K, 16), dtype=torch.uint8, device="cuda").view(code)
    s = torch.zeros(scale_rows, up(scale_cols, 16), dtype=torch.uint8, device="cuda")
    v = torch.zeros(rows, K, device="cuda")
    call(c, c.shape[1], s, s.shape[1], v)
    return c, s, v


@pytest.mark.parametrize("out", TYPES)
def test_experts_forward_and_backward(q, out):
    """Tokens in the order of their experts, a product, a gate, a product; then input and weight gradients from the same weights."""
    g, T, K, N, sizes = gen(11), 150, 300, 260, [70, 0, 129, 101]       # every token goes to two experts
    M, G = sum(sizes), len(sizes)
    off, at = offsets_of(sizes), [0] + torch.tensor(sizes).cumsum(0).tolist()
    index = (torch.randperm(M, generator=g, device="cuda") % T).to(torch.int64)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, w1, w2 = rand(T, K), rand(G, 2 * N, K), rand(G, K, N)

    def rows(t, code, idx=None):
        R, C = (len(idx), t.shape[1]) if idx is not None else t.shape
        return quantised(lambda c, l, s, ls, v: q.qnn_quantize_blocks_f8(t, R, C, C, c, l, s, ls, index=idx, src_rows=t.shape[0] if idx is not None else 0,
                                                                         values=v, ld_values=C), R, C, R, up(C, B) // B, code)

    def weight(w):
        parts = [quantised(lambda c, l, s, ls, v: q.qnn_quantize_tiles_f8(w[i], *w[i].shape, w.shape[2], c, l, s, ls, values=v, ld_values=w.shape[2]),
                           *w[i].shape, up(w.shape[1], B) // B, up(w.shape[2], B) // B, E4M3) for i in range(G)]
        return torch.stack([p[0].view(torch.uint8) for p in parts]).view(E4M3), torch.stack([p[1] for p in parts]), torch.stack([p[2] for p in parts])

    def columns(t, code):
        R = B * (M // B + G)
        return quantised(lambda c, l, s, ls, v: q.qnn_quantize_columns_f8(t, M, t.shape[1], t.shape[1], off, G, c, l, s, ls, values=v, ld_values=t.shape[1]),
                         R, t.shape[1], R // B, t.shape[1], code)

    def product(a, w, n, k, across=False):
        o = torch.zeros(M, n, dtype=out, device="cuda")
        before = q.qnn_launch_count()
        q.qnn_gemm_f8_grouped(a[0], a[0].shape[1], a[1], a[1].shape[1], w[0], w[0].shape[2], w[1], w[1].shape[2], off, G, M, n, k, o, n, b_transposed=across)
        assert q.qnn_launch_count() == before + 1
        for i in range(G):
            m = w[2][i].double()
            within(o[at[i]:at[i + 1]], a[2][at[i]:at[i + 1]].double(), m if across else m.t(), k)
        return o

    W1, W2 = weight(w1), weight(w2)
    a1 = rows(x, E4M3, index)
    assert torch.equal(a1[2], rows(x, E4M3)[2][index]), "an index that comes twice gives the same row twice"
    h = product(a1, W1, 2 * N, K).float()
    a2 = rows(torch.nn.functional.silu(h[:, :N]) * h[:, N:], E4M3)
    y = product(a2, W2, K, N)
    dy = rand(*y.shape)
    product(rows(dy, E5M2), W2, N, K, across=True)
    cy, cx = columns(dy, E5M2), columns(a2[2], E4M3)
    dw = torch.full((G, K, N), 7.0, dtype=out, device="cuda")
    q.qnn_gemm_f8_wgrad(cy[0], cy[0].shape[1], cy[1], cy[1].shape[1], cx[0], cx[0].shape[1], cx[1], cx[1].shape[1], off, G, M, K, N, dw, N)
    blk = 0
    for i, rows_i in enumerate(sizes):
        r = slice(blk * B, (blk + up(rows_i, B) // B) * B)
        blk += up(rows_i, B) // B
        a, b = cy[2][r].double(), cx[2][r].double()
        within(dw[i], a.t(), b, max(rows_i, 1))
        if out == torch.float32 and rows_i:
            # against differences: the loss sum(dy * (x w^T)) along a direction is linear, so its difference is the gradient's product with it
            d = rand(K, N).double()
            loss = lambda w: (a * (b @ w.t())).sum()
            slope, bound = (loss(d) - loss(-d)) / 2, ((a.abs().t() @ b.abs()) * d.abs()).sum() * rows_i * 2.0 ** -23
            assert (slope - (dw[i].double() * d).sum()).abs() <= bound + 1e-9 * slope.abs()


@pytest.mark.parametrize("across", [False, True], ids=["forward", "across"])
@pytest.mark.parametrize("M", [1, 16, 40, 130, 700])
def test_nan_scales_stay_in_their_rows_and_channels(q, M, across):
    g, N, K = gen(M), 300, 400
    a = Operand(g, M, K, E4M3, (1, B))
    w = Operand(g, K if across else N, N if across else K, E4M3, (B, B))
    a.scale[M // 2, 1] = 255
    if M > 1:
        w.scale[(2, 1) if across else (1, 2)] = 255                     # channels 128..255
    o = Guarded((M, N), torch.float32)
    q.qnn_gemm_f8(a.codes, a.ld, a.scale, a.lds, w.codes, w.ld, w.scale, w.lds, M, N, K, o.t, N, b_transposed=across)
    o.check()
    want = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    want[M // 2] = True
    if M > 1:
        want[:, 128:256] = True
    assert torch.equal(o.t.isnan(), want)


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("M,N", [(1, 5), (40, 300), (3000, 2000)])
def test_an_empty_reduction_gives_the_bias(q, M, N, out):
    c, s = torch.zeros(up(max(M, N), 16), 16, dtype=torch.uint8, device="cuda").view(E4M3), torch.zeros(up(max(M, N), 16), 16, dtype=torch.uint8, device="cuda")
    bias = torch.arange(N, device="cuda", dtype=torch.float32)
    for b in (bias, None):
        o = Guarded((M, N), out)
        q.qnn_gemm_f8(c, 16, s, 16, c, 16, s, 16, M, N, 0, o.t, N, bias=b)
        o.check()
        assert torch.equal(o.t, (bias if b is not None else bias * 0).to(out).expand(M, N))


def test_grouped_offsets_that_fall_or_leave_the_rows(q):
    g, M, N, K = gen(9), 300, 130, 200
    a = Operand(g, M, K, E4M3, (1, B))
    codes, scales, _ = weights(g, 4, N, K, E4M3)
    out = []
    for offs in ([-5, 200, 100, 900, 50], [0, 200, 200, 300, 300]):
        o = Guarded((M, N), torch.float32)
        t = torch.tensor(offs, dtype=torch.int64, device="cuda")
        q.qnn_gemm_f8_grouped(a.codes, a.ld, a.scale, a.lds, codes, codes.shape[2], scales, scales.shape[2], t, 4, M, N, K, o.t, N)
        o.check()
        out.append(o.t.clone())
    assert torch.equal(*out)


@pytest.mark.parametrize("M", [1, 40, 129, 700])
def test_products_captured_and_on_two_streams(q, M):
    g, N, K = gen(M), 512, 1024
    a, w = Operand(g, M, K, E4M3, (1, B)), Operand(g, N, K, E4M3, (B, B))
    outs = [torch.zeros(M, N, device="cuda") for _ in range(4)]
    call = lambda o: q.qnn_gemm_f8(a.codes, a.ld, a.scale, a.lds, w.codes, w.ld, w.scale, w.lds, M, N, K, o, N)
    call(outs[0])
    torch.cuda.synchronize()
    for s, o in zip([torch.cuda.Stream(), torch.cuda.Stream()], outs[1:3]):
        with torch.cuda.stream(s):
            call(o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[3])
    for _ in range(2):
        outs[3].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[0], o) for o in outs[1:]) and (outs[0] != 0).any()
