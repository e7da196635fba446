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
