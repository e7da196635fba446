"""How ``sqnn_moe_fp8`` may be called: layers of one inner value or one output, the status word, streams, workspaces of the exact size."""
import pytest
import torch

from paper_1905_10138_b200 import sqnn
from tests import fp8_helpers as F
from tests.test_moe_fp8 import call, check, layer, tokens_of

F32, BF16 = F.F32, F.BF16


def rows_apart(q, row):
    """The same 8-bit tensor with its rows `row` bytes apart, whatever its last dimensions are."""
    wide = torch.full((*q.shape[:-1], row), 0x7f, dtype=torch.uint8, device="cuda")
    wide[..., :q.shape[-1]] = q.view(torch.uint8)
    return wide.view(F.E4M3)[..., :q.shape[-1]]


@pytest.mark.gpu
@pytest.mark.parametrize("experts", [1, 5])
@pytest.mark.parametrize("hidden,inner,gu_row,down_row", [(64, 1, 80, 16), (1, 40, 32, 64), (1, 1, 48, 112), (200, 1, 224, 48)])
def test_rows_further_apart_where_there_is_one(experts, hidden, inner, gu_row, down_row):
    router, gu, gus, down, ds = layer(experts, hidden, inner, F32, 3)
    if hidden == 1:
        router.copy_(torch.arange(1, experts + 1, device="cuda")[:, None])
    lay, x = (router, rows_apart(gu, gu_row), gus, rows_apart(down, down_row), ds), tokens_of(3, hidden, F32, 4)
    top_k = min(2, experts)
    got = call(x, lay, top_k)
    check(x, lay, top_k, got)
    assert all(torch.equal(a, b) for a, b in zip(got, call(x, (router, gu, gus, down, ds), top_k)))


@pytest.mark.gpu
def test_gates_of_all_experts_before_their_ups():
    router, gu, gus, down, ds = layer(5, 64, 1, F32, 3)
    x = tokens_of(3, 64, F32, 4)
    apart = gu.view(torch.uint8).transpose(0, 1).contiguous().transpose(0, 1).view(F.E4M3)      # expert stride 64, G to U 320
    assert apart.stride(1) == 320
    assert all(torch.equal(a, b) for a, b in zip(call(x, (router, apart, gus, down, ds), 2), call(x, (router, gu, gus, down, ds), 2)))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,experts,top_k,hidden,inner,x_type", [(1, 64, 8, 512, 256, BF16), (5, 12, 3, 1000, 500, F32), (16, 32, 4, 768, 300, BF16),
                                                                      (64, 40, 4, 260, 130, F32), (29, 8, 7, 367, 1500, F32)])
def test_status_stream_and_a_workspace_of_the_exact_size(tokens, experts, top_k, hidden, inner, x_type):
    lay, x = layer(experts, hidden, inner, x_type, 5), tokens_of(tokens, hidden, x_type, 6)
    want = call(x, lay, top_k)
    router, gu, gus, down, ds = lay
    need = sqnn.sqnn_moe_workspace_bytes(tokens, top_k, inner)
    wide = torch.full((need + 512,), 0x5a, dtype=torch.uint8, device="cuda")
    y, status = torch.empty_like(x), torch.zeros(1, dtype=torch.int32, device="cuda")
    ids, probs = torch.empty((tokens, top_k), dtype=torch.int32, device="cuda"), torch.empty((tokens, top_k), device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        sqnn.sqnn_moe_fp8(x, router, top_k, True, gu, gus, down, ds, y, wide[:need], d_ids=ids, d_probs=probs, d_status=status, stream=stream)
    stream.synchronize()
    assert int(status.item()) == 0
    assert bool((wide[need:] == 0x5a).all())                       # nothing behind the workspace
    assert all(torch.equal(a, b) for a, b in zip((y, ids, probs), want))
