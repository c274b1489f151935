"""Forms of the 8-bit floating-point calls: without values, without offsets, captured, with rows far apart.  Compared bit for bit."""
import pytest
import torch

from test_gpu_f8_kernels import product
from test_gpu_f8_ops import B, E4M3, E5M2, TYPES, Operand, Out, check_out, gen, offsets_of, padded, q, ref_blocks, strided, up  # noqa: F401
from util import Guarded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", [E4M3, E5M2])
def test_quantisers_without_values(q, code, dtype):
    for rows, K in [(1, 1), (5, 100), (3, 256), (130, 1000), (2, 1025), (3, 4097), (300, 640)]:
        for ld, off in [(up(K, 8), 0), (K + 3, 1)]:
            x = strided(rows, K, ld, dtype, off, gen(rows + K), 3.0)
            o = Out(rows, K, rows, up(K, B) // B, code)
            q.qnn_quantize_blocks_f8(x, rows, K, ld, o.q, o.ldq, o.scale.t, o.lds)
            o.check(*ref_blocks(x.double(), 1, B, code), (1, B))
            o = Out(rows, K, up(rows, B) // B, up(K, B) // B, code)
            q.qnn_quantize_tiles_f8(x, rows, K, ld, o.q, o.ldq, o.scale.t, o.lds)
            o.check(*ref_blocks(x.double(), B, B, code), (B, B))
            blocks = rows // B + 1
            o = Out(blocks * B, K, blocks, K, code)
            q.qnn_quantize_columns_f8(x, rows, K, ld, None, 1, o.q, o.ldq, o.scale.t, o.lds)
            want, s = ref_blocks(padded(x.double(), [rows]), B, 1, code)
            o.check(want, s, (B, 1), rows=want.shape[0])


@pytest.mark.parametrize("M", [1, 64, 128, 129, 1000])
def test_weight_gradient_without_offsets(q, M):
    for n, (N, K) in enumerate([(128, 128), (300, 516), (1, 241)]):
        g = gen(M + N)
        rows = up(M, B)
        y, x = Operand(g, rows, N, E5M2, (B, 1)), Operand(g, rows, K, E5M2, (B, 1))
        for t in (y, x):
            t.codes.view(torch.uint8)[M:] = 0
            t.exact[M:] = 0
        o = Guarded((N, K), TYPES[n])
        q.qnn_gemm_f8_wgrad(y.codes, y.ld, y.scale, y.lds, x.codes, x.ld, x.scale, x.lds, None, 1, M, N, K, o.t, K)
        check_out(o, y.exact.t() @ x.exact)


def test_rows_before_the_first_offset_have_no_weight_gradient(q):
    sizes, first, N, K = [70, 0, 200], 150, 40, 100
    M, G = first + sum(sizes) + 11, len(sizes)
    g = gen(4)
    y, x = (torch.randint(-2, 3, (M, c), generator=g, device="cuda").float() for c in (N, K))
    off, blocks, made = offsets_of(sizes, first), M // B + G, []
    for t in (y, x):
        o = Out(blocks * B, t.shape[1], blocks, t.shape[1], E4M3)
        q.qnn_quantize_columns_f8(t, M, t.shape[1], t.shape[1], off, G, o.q, o.ldq, o.scale.t, o.lds)
        made.append(o)
    dw = Guarded((G * N, K), torch.float32)
    a, b = made
    q.qnn_gemm_f8_wgrad(a.q, a.ldq, a.scale.t, a.lds, b.q, b.ldq, b.scale.t, b.lds, off, G, M, N, K, dw.t, K)
    dw.check()
    at = first
    for i, n in enumerate(sizes):
        assert torch.equal(dw.t[i * N:(i + 1) * N], (y[at:at + n].double().t() @ x[at:at + n].double()).float())
        at += n


def test_a_step_captured_and_replayed_on_new_inputs(q):
    """Quantisers, products and weight gradient of a layer in one CUDA graph, beside another stream's calls on the same inputs."""
    M, N, K = 300, 200, 260
    g = gen(12)
    x, dy, w = (torch.zeros(*s, device="cuda") for s in ((M, K), (M, N), (N, K)))

    def buffers():
        u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
        z = lambda *s: torch.zeros(*s, device="cuda")
        rows = B * (M // B + 1)
        return dict(xq=u8(M, 272).view(E4M3), xs=u8(M, 16), wq=u8(N, 272).view(E4M3), ws=u8(16, 16), dq=u8(M, 208).view(E5M2), ds=u8(M, 16),
                    cy=u8(rows, 208).view(E5M2), cys=u8(rows // B, 208), cx=u8(rows, 272).view(E4M3), cxs=u8(rows // B, 272), y=z(M, N), dx=z(M, K), dw=z(N, K))

    def step(b):
        q.qnn_quantize_blocks_f8(x, M, K, K, b["xq"], 272, b["xs"], 16)
        q.qnn_quantize_tiles_f8(w, N, K, K, b["wq"], 272, b["ws"], 16)
        q.qnn_gemm_f8(b["xq"], 272, b["xs"], 16, b["wq"], 272, b["ws"], 16, M, N, K, b["y"], N)
        q.qnn_quantize_blocks_f8(dy, M, N, N, b["dq"], 208, b["ds"], 16)
        q.qnn_gemm_f8(b["dq"], 208, b["ds"], 16, b["wq"], 272, b["ws"], 16, M, K, N, b["dx"], K, b_transposed=True)
        q.qnn_quantize_columns_f8(dy, M, N, N, None, 1, b["cy"], 208, b["cys"], 208)
        q.qnn_quantize_columns_f8(x, M, K, K, None, 1, b["cx"], 272, b["cxs"], 272)
        q.qnn_gemm_f8_wgrad(b["cy"], 208, b["cys"], 208, b["cx"], 272, b["cxs"], 272, None, 1, M, N, K, b["dw"], K)

    captured, eager = buffers(), buffers()
    step(captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    side = torch.cuda.Stream()
    for seed in range(3):
        for t in (x, dy, w):
            t.copy_(torch.randint(-2, 3, t.shape, generator=g, device="cuda").float())
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            step(eager)
        torch.cuda.synchronize()
        X, D, W = x.double(), dy.double(), w.double()
        for b in (captured, eager):
            assert torch.equal(b["y"], (X @ W.t()).float()) and torch.equal(b["dx"], (D @ W).float()) and torch.equal(b["dw"], (D.t() @ X).float())


def test_rows_far_apart(q):
    """Elements more than 2^31 from the first one: inputs, codes, values and results with rows 2^30 and more apart."""
    far, rows, K, N = (1 << 30) + 16, 4, 200, 24
    g = gen(3)
    x = torch.empty(rows * far, dtype=torch.bfloat16, device="cuda").view(rows, far)
    x[:, :K] = torch.randint(-2, 3, (rows, K), generator=g, device="cuda").to(torch.bfloat16)
    codes = torch.full((rows * far,), 0xA5, dtype=torch.uint8, device="cuda").view(rows, far).view(E4M3)
    scale = torch.zeros(rows, 16, dtype=torch.uint8, device="cuda")
    values = torch.empty(rows * far, dtype=torch.bfloat16, device="cuda").view(rows, far)
    want, s = ref_blocks(x[:, :K].double(), 1, B, E4M3)
    q.qnn_quantize_blocks_f8(x, rows, K, far, codes, far, scale, 16, values=values, ld_values=far)
    assert torch.equal(codes[:, :K].double(), want) and torch.equal(scale[:, :2], s) and torch.equal(values[:, :K], x[:, :K])
    w = Operand(g, N, K, E4M3, (B, B))
    out = torch.empty(rows * far, dtype=torch.bfloat16, device="cuda").view(rows, far)
    q.qnn_gemm_f8(codes, far, scale, 16, w.codes, w.ld, w.scale, w.lds, rows, N, K, out, far)
    exact = x[:, :K].double() @ w.exact.t()
    assert torch.equal(out[:, :N], exact.float().to(torch.bfloat16))
    # as weights: forward and across
    ws = torch.zeros(1, 16, dtype=torch.uint8, device="cuda")
    q.qnn_quantize_tiles_f8(x, rows, K, far, codes, far, ws, 16, values=values, ld_values=far)
    assert torch.equal(values[:, :K], x[:, :K])
    for across, (m, n, k) in ((False, (5, rows, K)), (True, (5, K, rows))):
        a = Operand(g, m, k, E4M3, (1, B))
        o = product(q, a, type("W", (), dict(codes=codes, ld=far, scale=ws, lds=16)), m, n, k, torch.float32, n, across)
        check_out(o, a.exact @ (x[:, :K].double() if across else x[:, :K].double().t()))
    del values, codes
    cq, cs = torch.zeros(2 * B, 208, dtype=torch.uint8, device="cuda").view(E4M3), torch.zeros(2, 208, dtype=torch.uint8, device="cuda")
    q.qnn_quantize_columns_f8(x, rows, K, far, None, 1, cq, 208, cs, 208)
    y = Operand(g, B, rows, E4M3, (B, 1))
    y.codes.view(torch.uint8)[rows:] = 0
    q.qnn_gemm_f8_wgrad(y.codes, y.ld, y.scale, y.lds, cq, 208, cs, 208, None, 1, rows, rows, K, out, far)
    assert torch.equal(out[:, :K], (y.exact[:rows].t() @ x[:, :K].double()).float().to(torch.bfloat16))


@pytest.mark.parametrize("out", TYPES)
def test_an_empty_reduction_by_group_gives_the_groups_bias(q, out):
    sizes, first, N = [40, 0, 300, 1], 2, 200
    M, G = first + sum(sizes) + 5, len(sizes)
    c, s = torch.zeros(512, 16, dtype=torch.uint8, device="cuda").view(E4M3), torch.zeros(512, 16, dtype=torch.uint8, device="cuda")
    bias = torch.arange(G * N, device="cuda", dtype=torch.float32).view(G, N)
    for b in (bias, None):
        o = Guarded((M, N), out)
        q.qnn_gemm_f8_grouped(c, 16, s, 16, c, 16, s, 16, offsets_of(sizes, first), G, M, N, 0, o.t, N, bias=b)
        o.check()
        at = first
        for i, n in enumerate(sizes):
            assert torch.equal(o.t[at:at + n], ((b if b is not None else 0 * bias)[i]).to(out).expand(n, N))
            at += n
        for r in (slice(0, first), slice(at, M)):
            assert (o.t[r].view(torch.uint8) == 0xA5).all()


def test_products_beside_one_another_on_three_streams(q):
    """Products of every kind at once: clusters and pairs of one stream's call wait for SMs, shared and tensor memory of the other's."""
    g, jobs = gen(8), []
    for M, N, K in [(1, 4096, 4096), (250, 1030, 4700), (2000, 2000, 600), (7, 2000, 4200), (950, 520, 2300), (4000, 2100, 600), (40, 3000, 260)]:
        a, w = Operand(g, M, K, E4M3, (1, B)), Operand(g, N, K, E4M3, (B, B))
        jobs.append((a, w, M, N, K, (a.exact @ w.exact.t()).float()))
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[torch.zeros(j[2], j[3], device="cuda") for j in jobs] for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for n, (st, out) in enumerate(zip(streams, outs)):
            with torch.cuda.stream(st):
                for i in range(len(jobs)):
                    a, w, M, N, K, _ = jobs[(i * (n + 1)) % len(jobs)]
                    q.qnn_gemm_f8(a.codes, a.ld, a.scale, a.lds, w.codes, w.ld, w.scale, w.lds, M, N, K, out[(i * (n + 1)) % len(jobs)], N)
    torch.cuda.synchronize()
    for out in outs:
        for o, j in zip(out, jobs):
            assert torch.equal(o, j[5])
