"""The 8-bit operators as a block of a model calls them, in place where they may be, captured into one graph."""
import pytest
import torch

from paper_1905_10138_b200 import sqnn
from tests import fp8_helpers as F
from tests import test_fp8_matmul as product
from tests import test_moe_fp8 as mixture
from tests import test_rmsnorm_fp8 as norm

F32, BF16 = F.F32, F.BF16


@pytest.mark.gpu
@pytest.mark.parametrize("n", [777, 4096, 20000])
@pytest.mark.parametrize("kind", [BF16, F32])
def test_norm_over_its_inputs(n, kind):
    xs, r, w = norm.inputs(7, n, kind, kind, kind, n)
    q, s, d_w = F.rows16((7, n), "cuda"), torch.empty((7, F.blocks(n)), device="cuda"), w.cuda()
    d_x, d_r = xs.cuda(), r.cuda()
    sqnn.sqnn_rmsnorm_fp8(d_x, d_w, 1e-6, q, s, d_r, d_x)          # h over x
    norm.check(xs, w, 1e-6, r, (d_x.cpu(), None, q.cpu(), s.cpu()))
    d_x = xs.cuda()
    sqnn.sqnn_rmsnorm_fp8(d_x, d_w, 1e-6, q, s, None, None, d_x)   # y over x
    norm.check(xs, w, 1e-6, None, (None, d_x.cpu(), q.cpu(), s.cpu()), kind)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 5, 40])
def test_a_block_in_one_graph(tokens):
    """Norm, product, norm with the residual in place, mixture: replayed with other inputs it gives what the calls give."""
    n = 1024
    router, gu, gus, down, ds = mixture.layer(16, n, 256, BF16, 3)
    w, ws, _, _ = product.operands(n, n, 1, 4)
    g = torch.Generator().manual_seed(tokens)

    def rows():
        return torch.randn((tokens, n), generator=g).to(BF16).cuda()

    x, residual, weight = rows(), rows(), (torch.rand(n, generator=g) + 0.5).to(BF16).cuda()
    q, s = F.rows16((tokens, n), "cuda"), torch.empty((tokens, F.blocks(n)), device="cuda")
    h, normed, y = (torch.empty((tokens, n), dtype=BF16, device="cuda") for _ in range(3))
    mid = torch.empty((tokens, n), device="cuda")
    workspace = torch.empty(sqnn.sqnn_moe_workspace_bytes(tokens, 4, 256), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def block():
        sqnn.sqnn_rmsnorm_fp8(x, weight, 1e-6, q, s, residual, h)
        sqnn.sqnn_fp8_matmul(w, ws, q, s, mid, status)
        sqnn.sqnn_rmsnorm_fp8(mid, weight, 1e-6, None, None, h, h, normed)
        sqnn.sqnn_moe_fp8(normed, router, 4, True, gu, gus, down, ds, y, workspace, d_status=status)

    def outputs():
        torch.cuda.synchronize()
        got = [t.clone() for t in (q.view(torch.uint8), s, mid, h, normed, y)]
        for t in (q.view(torch.uint8), s, mid, h, normed, y):
            t.zero_()
        return got

    block()
    first = outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for _ in range(3):
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(first, outputs()))
    x.copy_(rows())
    graph.replay()
    second = outputs()
    block()
    assert all(torch.equal(a, b) for a, b in zip(second, outputs())) and not torch.equal(first[5], second[5])
    _, _, want_q, want_s = F.rmsnorm(x.cpu(), weight.cpu(), 1e-6, residual.cpu())
    norm.same(second[0].view(F.E4M3).float().cpu(), want_q)
    norm.same(second[1].cpu(), want_s)
    ids, probs = torch.empty((tokens, 4), dtype=torch.int32, device="cuda"), torch.empty((tokens, 4), device="cuda")
    sqnn.sqnn_moe_fp8(second[4], router, 4, True, gu, gus, down, ds, y, workspace, ids, probs, status)
    torch.cuda.synchronize()
    assert torch.equal(y, second[5]) and int(status.item()) == 0
    mixture.check(second[4], (router, gu, gus, down, ds), 4, (y, ids, probs))
