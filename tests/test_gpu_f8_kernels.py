"""Every kernel that products of 8-bit floating-point codes are dispatched to.  Inputs are made so that sums are exact (see
test_gpu_f8_ops.py), and results are compared bit for bit."""
import pytest
import torch

from test_gpu_f8_ops import B, E4M3, E5M2, TYPES, Operand, check_out, gen, offsets_of, q, up, weights  # noqa: F401
from util import Guarded

pytestmark = pytest.mark.gpu

# a size for every instance, and for the pair of CTAs (width 256) one each with tiles of 160, 224 and 256 columns (the accumulators
# apart and sharing columns), a second half beyond the channels, and more than 16 chunks of tokens
INSTANCES = [(1, 300, 1000), (9, 260, 2000), (7, 200, 4200), (40, 300, 260), (5000, 300, 140), (10000, 100, 300), (400, 300, 1800), (300, 200, 2400),
             (250, 100, 4700), (250, 130, 8000), (950, 520, 2300), (400, 520, 2100), (450, 140, 4000), (1600, 700, 2300), (2000, 2000, 600),
             (4000, 2100, 600), (10000, 700, 1030)]


def test_instances_are_all_of_them(q):
    every = {(16, 2), (16, 4), (16, 8), (32, 1), (64, 1), (128, 1), (256, 1)} | {(w, s) for w in (64, 128) for s in (2, 4, 8)}
    reached = {q.qnn_gemm_f8_kernel(M, N, K)[:2] for M, N, K in INSTANCES}
    assert reached == every, (every - reached, reached - every)
    assert {q.qnn_gemm_f8_kernel(M, N, K)[2] for M, N, K in INSTANCES if q.qnn_gemm_f8_kernel(M, N, K)[0] == 256} == {160, 224, 256}
    for none in ((0, 5, 5), (5, 0, 5), (5, 5, -1), (5, 5, 5, -1), (5, 5, 5, 1025), ((1 << 30) + 1, 5, 5)):
        assert q.qnn_gemm_f8_kernel(*none) == (0, 0, 0)


def product(q, a, w, M, N, K, out, ldo, across, bias=None):
    o = Guarded((M, ldo), out)
    q.qnn_gemm_f8(a.codes, a.ld, a.scale, a.lds, w.codes, w.ld, w.scale, w.lds, M, N, K, o.t, ldo, bias=bias, b_transposed=across)
    return o


@pytest.mark.parametrize("across", [False, True], ids=["forward", "across"])
@pytest.mark.parametrize("M,N,K", INSTANCES)
def test_product_instances(q, M, N, K, across):
    """Rows that leave as bulk stores (N a multiple of 8) and rows of every alignment (N odd), all types."""
    for odd in (False, True):
        n = N | 1 if odd else up(N, 8)
        assert q.qnn_gemm_f8_kernel(M, n, K) == q.qnn_gemm_f8_kernel(M, N, K)
        for i, out in enumerate(TYPES):
            g = gen(M + n + K + i)
            a = Operand(g, M, K, (E4M3, E5M2, E5M2)[i], (1, B), pad=16 * (i % 2))
            w = Operand(g, K if across else n, n if across else K, (E4M3, E4M3, E5M2)[i], (B, B), pad=16 * (i // 2))
            bias = torch.randint(-8, 9, (n,), generator=g, device="cuda").float() if i else None
            o = product(q, a, w, M, n, K, out, n, across, bias)
            want = a.exact @ (w.exact if across else w.exact.t())
            check_out(o, want + bias.double() if bias is not None else want)


# more than 64 tiles for every CTA (or pair): both halves of the tiles on their way to its warps are filled again
@pytest.mark.parametrize("M,N,K,width", [(1, 1300000, 128, 32), (700000, 128, 128, 64), (70000, 4864, 256, 128), (70000, 4864, 600, 256)])
def test_many_tiles_a_worker(q, M, N, K, width):
    assert q.qnn_gemm_f8_kernel(M, N, K)[0] == width
    g = gen(M + N)
    for across in (False, True):
        a, w = Operand(g, M, K, E4M3, (1, B)), Operand(g, K if across else N, N if across else K, E4M3, (B, B))
        o = product(q, a, w, M, N, K, torch.bfloat16, N, across)
        o.check()
        other = w.exact if across else w.exact.t()
        for r in range(0, M, 10000):
            want = a.exact[r:r + 10000] @ other
            assert torch.equal(o.t[r:r + 10000], want.float().to(torch.bfloat16)), r
        del o, a, w, other, want


# few rows, none and many; the pair of CTAs has eight columns each of a group of five rows
UNEVEN = [5, 4100, 0, 2500, 33, 130]


@pytest.mark.parametrize("across", [False, True], ids=["forward", "across"])
@pytest.mark.parametrize("N,K,sizes,width", [(1300, 1000, UNEVEN, 256), (1307, 1000, UNEVEN, 256), (640, 516, [2000, 3, 0, 300, 1, 129, 3900, 18], 128),
                                             (300, 516, [700, 0, 1900, 400], 64)])
def test_grouped_instances(q, N, K, sizes, width, across):
    G, first, behind = len(sizes), 3, 40
    M = first + sum(sizes) + behind
    assert q.qnn_gemm_f8_kernel(M, N, K, G) == (width, 1, width)
    for i, out in enumerate(TYPES):
        g = gen(N + i)
        a = Operand(g, M, K, (E4M3, E5M2, E5M2)[i], (1, B))
        codes, scales, ws = weights(g, G, K if across else N, N if across else K, (E4M3, E4M3, E5M2)[i])
        bias = torch.randint(-8, 9, (G, N), generator=g, device="cuda").float() if i else None
        o = Guarded((M, N), out)
        q.qnn_gemm_f8_grouped(a.codes, a.ld, a.scale, a.lds, codes, codes.shape[2], scales, scales.shape[2], offsets_of(sizes, first), G, M, N, K, o.t, N,
                              bias=bias, b_transposed=across)
        o.check()
        at = first
        for n, rows in enumerate(sizes):
            want = a.exact[at:at + rows] @ (ws[n].exact if across else ws[n].exact.t())
            if bias is not None:
                want = want + bias[n].double()
            assert torch.equal(o.t[at:at + rows], want.to(torch.float32).to(out)), n
            at += rows
        for r in (slice(0, first), slice(at, M)):
            assert (o.t[r].view(torch.uint8) == 0xA5).all(), "rows of no group are left as they were"
