"""The 8-bit floating-point calls with many groups, offsets that fall or leave the rows among them.  Sums are exact and compared bit
for bit."""
import pytest
import torch

from test_gpu_f8_ops import B, E4M3, Operand, Out, gen, offsets_of, padded, q, ref_blocks, weights  # noqa: F401
from util import Guarded

pytestmark = pytest.mark.gpu


def few_rows(groups, seed):
    """Mostly none to two rows a group, and some larger groups next to where a warp's or a batch's share of the offsets ends."""
    g = torch.Generator().manual_seed(seed)
    sizes = torch.randint(0, 3, (groups,), generator=g).tolist()
    for at, n in ((31, 40), (32, 7), (63, 130), (64, 3), (95, 300), (96, 129), (97, 64), (191, 20), (192, 21), (groups - 1, 5)):
        if at < groups:
            sizes[at] = n
    return sizes


def held(offsets, M):
    """What offsets that fall or leave 0..M are taken as."""
    return offsets.clamp(0, M).cummax(0).values


def broken(offsets, M):
    """Offsets that fall, or leave 0..M, at the ends of a warp's and of a batch's share, and what they are held to."""
    o = offsets.clone()
    G = len(o) - 1
    o[0] = -7
    for at in (30, 31, 32, 33, 63, 64, 65, 94, 95, 97, 98, 190, 193, 288):
        if at < G:
            o[at] = (0, -5, o[at - 3], o[at] // 2)[at % 4]
    o[G - 1] = M + 1000
    o[G] = 3
    return o, held(o, M)


@pytest.mark.parametrize("fall", [False, True], ids=["rising", "falling"])
@pytest.mark.parametrize("groups", [97, 200, 1024])
def test_many_groups_product(q, groups, fall):
    N = K = 128
    sizes = few_rows(groups, groups)
    M = sum(sizes) + 9
    g = gen(groups)
    a = Operand(g, M, K, E4M3, (1, B))
    codes, scales, ws = weights(g, groups, N, K, E4M3)
    offs = offsets_of(sizes, 4)
    given, real = broken(offs.cpu(), M) if fall else (offs.cpu(), offs.cpu())
    o = Guarded((M, N), torch.float32)
    before = o.t.clone()
    q.qnn_gemm_f8_grouped(a.codes, a.ld, a.scale, a.lds, codes, K, scales, scales.shape[2], given.cuda(), groups, M, N, K, o.t, N)
    o.check()
    want = before.double()
    for i in range(groups):
        r = slice(int(real[i]), int(real[i + 1]))
        if r.stop > r.start:
            want[r] = a.exact[r] @ ws[i].exact.t()
    assert torch.equal(o.t.view(torch.int32), want.float().view(torch.int32))


@pytest.mark.parametrize("fall", [False, True], ids=["rising", "falling"])
@pytest.mark.parametrize("groups", [97, 200, 1024])
def test_many_groups_columns_and_weight_gradient(q, groups, fall):
    """The column quantiser's blocks and the weight gradients computed from them."""
    N = K = 32
    sizes = few_rows(groups, groups + 1)
    M = sum(sizes) + 9
    g = gen(groups)
    offs = offsets_of(sizes, 4).cpu()
    given, real = broken(offs, M) if fall else (offs, offs)
    sizes, first = (real[1:] - real[:-1]).tolist(), int(real[0])
    y, x = (torch.randint(-2, 3, (M, c), generator=g, device="cuda").float() for c in (N, K))
    blocks = M // B + groups
    made = []
    for t in (y, x):
        o = Out(blocks * B, t.shape[1], blocks, t.shape[1], E4M3)
        q.qnn_quantize_columns_f8(t, M, t.shape[1], t.shape[1], given.cuda(), groups, o.q, o.ldq, o.scale.t, o.lds)
        want, s = ref_blocks(padded(t.double(), sizes, first), B, 1, E4M3)
        o.check(want, s, (B, 1), rows=want.shape[0])
        made.append(o)
    dw = Guarded((groups * N, K), torch.float32)
    a, b = made
    q.qnn_gemm_f8_wgrad(a.q, a.ldq, a.scale.t, a.lds, b.q, b.ldq, b.scale.t, b.lds, given.cuda(), groups, M, N, K, dw.t, K)
    dw.check()
    want = torch.stack([y[first + sum(sizes[:i]):][:n].double().t() @ x[first + sum(sizes[:i]):][:n].double() for i, n in enumerate(sizes)])
    assert torch.equal(dw.t.view(groups, N, K), want.float())
