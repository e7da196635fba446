"""Which experts ``sqnn_moe_fp8`` chooses where 32 bits cannot tell their logits apart: the choice is that of the exact logits."""
import pytest
import torch

from tests import fp8_helpers as F
from tests.test_moe_fp8 import call, layer, tokens_of

F32, BF16 = F.F32, F.BF16


def exact_choice(x, router, top_k):
    logits = x.double() @ router.double().T
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    return order.indices[:, :top_k], order.values


def near_ties(tokens, experts, hidden, x_type, seed, groups=1):
    """Logits that differ in their last bits only: a common part of about `hidden`, and k 2^-22 (bf16) or k 2^-26 (fp32) with another k per expert, in a column
    whose activation is 1.  All numbers and, in 64 bits, all sums are exact.  More than one group: logits of a group are near one another, groups are far apart."""
    g = torch.Generator().manual_seed(seed)
    x = (1 + torch.randint(0, 128, (tokens, hidden), generator=g) / 128.0)
    common = (1 + torch.randint(0, 128, (groups, hidden), generator=g) / 128.0)
    common[:, hidden // 2:] *= -1                                  # (the sum itself may be anything)
    router = common[torch.arange(experts) % groups].clone()
    router[:, hidden // 3] = 0
    unit = 2.0 ** -22 if x_type == BF16 else 2.0 ** -26
    router[:, hidden // 3] = (torch.randperm(experts, generator=g) % 250 + 1) * unit
    x[:, hidden // 3] = 1
    return x.to(x_type).cuda(), router.to(x_type).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
@pytest.mark.parametrize("tokens,experts,top_k,hidden,groups", [(1, 24, 4, 512, 1), (4, 60, 8, 509, 5), (7, 12, 12, 1000, 3), (18, 128, 7, 640, 9), (64, 250, 16, 256, 40),
                                                                (33, 6, 2, 2048, 1), (2, 250, 1, 96, 1), (9, 64, 5, 1003, 64)])
def test_the_choice_is_that_of_the_exact_logits(tokens, experts, top_k, hidden, groups, x_type):
    x, router = near_ties(tokens, experts, hidden, x_type, tokens + experts, groups)
    lay = (router, *layer(experts, hidden, 64, x_type, 3)[1:])
    want, _ = exact_choice(x, router, top_k)
    first = call(x, lay, top_k)
    assert torch.equal(first[1].long(), want)
    assert all(torch.equal(a, b) for a, b in zip(call(x, lay, top_k), first))


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
@pytest.mark.parametrize("tokens,experts,top_k", [(3, 20, 5), (17, 130, 6)])
@pytest.mark.parametrize("x_scale,router_scale", [(1e-38, 1e-4), (1e-36, 1e-8), (1e-38, 1e-30), (1e25, 1e30), (1e-30, 1.0), (3e37, 1e-3)])
def test_products_beyond_the_range_of_32_bits(tokens, experts, top_k, x_scale, router_scale, x_type):
    g = torch.Generator().manual_seed(9)
    x = (torch.randn((tokens, 600), generator=g) * x_scale).to(x_type).cuda()
    router = (torch.randn((experts, 600), generator=g) * router_scale).to(x_type).cuda()
    lay = (router, *layer(experts, 600, 32, x_type, 4)[1:])
    want, logits = exact_choice(x, router, top_k)
    _, ids, probs = call(x, lay, top_k)
    assert torch.equal(ids.long(), want)
    # a share: the exponential of a difference of logits, each within 2^-20 of the sum of magnitudes (2^-16 here), over a sum of such
    p = torch.softmax(logits[:, :top_k], 1)
    exponent = 2.0 ** -16 * (x.double().abs() @ router.double().abs().T).amax(1, keepdim=True)
    off = (probs.double() - p).abs()
    assert bool(((off <= (torch.expm1(torch.clamp(4 * exponent, max=700.0)) + 64 * 2.0 ** -24) * p + 1e-40) | (exponent > 1)).all())
    assert bool(torch.isfinite(probs).all()) and bool(((probs.sum(1) - 1).abs() < 1e-5).all())


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
@pytest.mark.parametrize("hidden", [64, 640, 1024])
def test_what_sums_of_a_few_products_cut_off(hidden, x_type):
    """Many small products beside a large one: each vanishes in a sum of 16 (or of 4), together they decide."""
    experts, small = 9, 2.0 ** -26 * 1.9921875
    router = torch.zeros((experts, hidden))
    router[:, 0::4] = (torch.arange(hidden // 4) % 16 < 4).float() if x_type == BF16 else 1.0
    many = router[4].clone()
    many[many == 0] = small
    router[4] = many                                               # the largest sum, but not to 32 bits
    count = int((many == small).sum())
    step = 2.0 ** -20 if x_type == BF16 else 2.0 ** -22
    for e in (2, 6, 8):                                            # as much as 32 bits show, and less than `many`
        room = int(count * small * 0.9 / step)
        router[e, (torch.nonzero(router[e] == 1).flatten() + 1)[:room]] = step
    x = torch.ones((3, hidden))
    x[1] *= -2
    x[2] *= 2.0 ** -20
    x, router = x.to(x_type).cuda(), router.to(x_type).cuda()
    lay = (router, *layer(experts, hidden, 64, x_type, 7)[1:])
    want, _ = exact_choice(x, router, 5)
    assert int(want[0, 0]) == 4
    assert torch.equal(call(x, lay, 5)[1].long(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
@pytest.mark.parametrize("tokens,experts,top_k,hidden", [(1, 64, 8, 2048), (9, 40, 16, 1003), (30, 128, 4, 4096)])
@pytest.mark.parametrize("renormalize", [True, False])
def test_shares(tokens, experts, top_k, hidden, renormalize, x_type):
    """With eps = 2^-24 and A the sum of a logit's products' magnitudes.  bf16: an MMA instruction adds 16 exact products, cut off below 2^-25 of the largest, and
    cuts its sum to 24 bits: (16 / 2 + 2) eps of their magnitudes; two additions make a sum of 64: 12 eps A.  fp32: eight fused multiply-adds, 8 eps A.  The rest is
    in 64 bits.  A difference of two logits has two such errors and a rounding, no more than 2 eps A.  A share is the exponential of one (expf: 2 units in the last
    place, 4 eps) over a sum of such (in fp32: one addition for each that a lane holds, five to join them, `experts` / 32 + 6), and a division."""
    eps = 2.0 ** -24
    lay, x = layer(experts, hidden, 32, x_type, 11), tokens_of(tokens, hidden, x_type, 12)
    x[:, 5] *= 20
    want, logits = exact_choice(x, lay[0], top_k)
    _, ids, probs = call(x, lay, top_k, renormalize)
    assert torch.equal(ids.long(), want)
    p = torch.softmax(logits[:, :top_k] if renormalize else logits, 1)[:, :top_k]
    total = (x.double().abs() @ lay[0].double().abs().T).amax(1, keepdim=True)
    exponent = (2 * (12 if x_type == BF16 else 8) + 2) * eps * total
    off = (probs.double() - p).abs()
    assert bool((off <= (2 * exponent + (2 * 4 + experts / 32 + 6 + 2) * eps) * p + 1e-40).all()), float((off / p).max())


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
def test_what_is_not_finite_leaves_the_rest_of_the_choice(x_type):
    x, router = near_ties(6, 40, 512, x_type, 5, 4)
    x[2, 9] = float("nan")
    x[4] = 0                                                       # all logits equal: the lowest indices
    router[7, 3] = float("nan")
    router[11, 500] = float("inf")
    router[13, 200] = float("-inf")
    lay = (router, *layer(40, 512, 64, x_type, 6)[1:])
    _, ids, _ = call(x, lay, 6)
    logits = x.double() @ router.double().T
    logits[torch.isnan(logits)] = float("inf")                     # NaN counts as the largest ..
    key = logits.clone()
    key[:, 11] = torch.where(logits[:, 11] == float("inf"), torch.finfo(torch.float64).max, logits[:, 11])     # .. above infinity
    key[:, 7] = float("inf")
    want = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :6]
    rows = [0, 1, 3, 5]
    assert torch.equal(ids.long()[rows], want[rows])
    assert ids[2].tolist() == [0, 1, 2, 3, 4, 5]
    assert ids[4].tolist() == [7, 11, 13, 0, 1, 2]                 # 0 x infinity is NaN


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
def test_routers_of_equal_rows_and_of_zeros(x_type):
    x = tokens_of(5, 300, x_type, 8)
    lay = layer(33, 300, 64, x_type, 9)
    router = lay[0]
    router[20:] = router[:13]                                      # each of thirteen rows twice
    want, _ = exact_choice(x, router, 8)
    assert torch.equal(call(x, lay, 8)[1].long(), want)
    router.zero_()
    _, ids, probs = call(x, lay, 8)
    assert bool((ids == torch.arange(8, dtype=torch.int32, device="cuda")).all()) and bool((probs == 0.125).all())
