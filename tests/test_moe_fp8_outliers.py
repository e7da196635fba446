"""``sqnn_moe_fp8`` for tokens whose largest activation lies in one place: the warps that share a token's columns must all find it, or the
activations are scaled too far up and leave the range of their pieces.  Tolerances as in ``test_moe_fp8``."""
import pytest
import torch

from tests import fp8_helpers as F
from tests.test_moe_fp8 import call, check, layer, tokens_of

F32, BF16 = F.F32, F.BF16


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
@pytest.mark.parametrize("tokens,experts,top_k,hidden,inner", [(1, 6, 2, 2048, 256), (5, 12, 3, 1000, 200), (8, 60, 2, 520, 128), (20, 40, 4, 768, 96)])
def test_the_largest_activation_in_one_place(tokens, experts, top_k, hidden, inner, x_type):
    lay, base = layer(experts, hidden, inner, x_type, tokens + hidden), tokens_of(tokens, hidden, x_type, 31)
    for column in (0, hidden // 16, hidden // 2 + 1, hidden - 1):
        x = base.clone()
        x[:, column] = 2.0 ** 9                                    # fp16 pieces end at 2^16: a scale from the rest (2^13 and up) is too large
        got = call(x, lay, top_k)
        check(x, lay, top_k, got)
        for _ in range(5):
            assert all(torch.equal(a, b) for a, b in zip(call(x, lay, top_k), got))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,experts,top_k,hidden,inner,x_type", [(64, 256, 16, 256, 64, BF16), (32, 512, 16, 192, 48, F32), (1, 512, 16, 128, 32, BF16)])
def test_weights_come_after_the_choice(tokens, experts, top_k, hidden, inner, x_type):
    """The weights' copies go where the logits were, which the choice of experts writes to until it is made: many logits and the most choices, call after call."""
    lay, x = layer(experts, hidden, inner, x_type, 41), tokens_of(tokens, hidden, x_type, 42)
    first = call(x, lay, top_k)
    check(x, lay, top_k, first)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(call(x, lay, top_k), first))


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
@pytest.mark.parametrize("hidden,inner", [(520, 96), (2048, 300)])
def test_inner_values_beyond_fp32_are_infinite(hidden, inner, x_type):
    """Positive weights throughout: y is infinite, not NaN, where gate and up are finite and their product is not."""
    router, gu, gus, down, ds = layer(5, hidden, inner, x_type, 51)
    for w in (gu, down):
        w.view(torch.uint8).bitwise_and_(0x7f).clamp_(min=8)       # no zeros: 0 x infinity is NaN
    lay = (router, gu, gus, down, ds)
    x = tokens_of(4, hidden, x_type, 52).abs()
    x[1] *= 1e25
    y, _, probs = call(x, lay, 1)
    assert bool((probs == 1).all()) and bool((y[1] == float("inf")).all())
    rest = [0, 2, 3]
    check(x[rest], lay, 1, call(x[rest], lay, 1))
    assert all(torch.equal(y[t], v) for t, v in zip(rest, call(x[rest], lay, 1)[0]))


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
def test_small_activations_beside_a_large_one_that_weighs_nothing(x_type):
    """Activations are left with 2^-39 of the token's largest off (and 2^-23 of themselves): the largest is 2^20 and its weights are zero."""
    hidden, inner, top_k = 640, 128, 2
    router, gu, gus, down, ds = layer(4, hidden, inner, x_type, 61)
    router[:, 100] = 0
    gu[..., 100] = 0
    x = tokens_of(3, hidden, x_type, 62)
    x[:, 100] = 2.0 ** 20
    y, ids, probs = call(x, (router, gu, gus, down, ds), top_k)
    xd = x.double()
    off = torch.maximum(2.0 ** -23 * xd.abs(), torch.full_like(xd, 2.0 ** -39 * 2.0 ** 20)) if x_type == F32 else torch.zeros_like(xd)
    s_h, s_i = (158 + hidden / 64) * 2.0 ** -24, (158 + inner / 64) * 2.0 ** -24      # sums of a layer: see test_moe_fp8
    for t in range(3):
        ref, tol = torch.zeros(hidden, dtype=torch.float64, device="cuda"), torch.zeros(hidden, dtype=torch.float64, device="cuda")
        for k in range(top_k):
            e, p = int(ids[t, k]), float(probs[t, k])
            wg, wu, wd = F.weight_values(gu[e, 0], gus[e, 0]), F.weight_values(gu[e, 1], gus[e, 1]), F.weight_values(down[e], ds[e])
            a, b = wg @ xd[t], wu @ xd[t]
            da, db = wg.abs() @ (s_h * xd[t].abs() + off[t]), wu.abs() @ (s_h * xd[t].abs() + off[t])
            silu = a * torch.sigmoid(a)
            v = silu * b
            dv = 1.1 * da * (b.abs() + db) + silu.abs() * db + 10 * 2.0 ** -24 * v.abs()
            ref += p * (wd @ v)
            tol += p * (wd.abs() @ (dv + (s_i + 40 * 2.0 ** -24) * v.abs()))
        if x_type == BF16:
            tol += F.HALF_STEP[BF16] * (ref.abs() + tol)
        assert bool(((y[t].double() - ref).abs() <= tol).all())
