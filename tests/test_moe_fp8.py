"""``sqnn_moe_fp8`` against its definition in 64 bits.

Tolerance.  eps = 2^-24.  A sum over `n` columns: weights are exact, activations are left with 2^-22 (fp32) or nothing (bf16) off; a chunk of
64 columns is four MMA instructions (twice that with two pieces) of 16 products each, at most 17 units per instruction where every addend keeps 25 bits, 136 in
all, then two roundings per chunk and up to 16 for the warps' parts: s(n) = (4 + 136 + 2 + n / 64 + 16) eps of the sum of magnitudes.  So gate and up are off by
s(hidden) A with A their sums of magnitudes.  silu has a slope of at most 1.1 and is itself off by 8 eps (expf 2 ulp, an addition, a division and a product), so the inner
values are off by d = 1.1 s A_gate |up| + |silu| s A_up + 10 eps |inner|.  y: sum p |D| d + s(inner) sum p |D| |inner| + 16 eps of that (shares: expf, sum, division; up to
top_k and 16 additions), and half a step of y for bf16.

Shares: eight fused multiply-adds in fp32 leave a logit off by at most 8 eps L with L = sum |x| |r| (each rounds a partial sum that is no larger); the difference to the
largest logit has two such errors and one rounding, at most 2 eps L: 18 eps L in the exponent.  A share is such an exponential over a sum of them, so it is
off by 36 eps L of itself beside its own roundings, and y's terms with it."""
import ctypes

import pytest
import torch

from paper_1905_10138_b200 import sqnn
from tests import fp8_helpers as F

F32, BF16 = F.F32, F.BF16
EPS = 2.0 ** -24


def layer(experts, hidden, inner, x_type, seed):
    g = torch.Generator().manual_seed(seed)
    router = (torch.randn((experts, hidden), generator=g) * 2 / hidden ** 0.5).to(x_type).cuda()
    gu, down = F.random_fp8((experts, 2, inner, hidden), g, "cuda"), F.random_fp8((experts, hidden, inner), g, "cuda")
    # e4m3 of all magnitudes has an rms of about 90
    gus = (0.01 / hidden ** 0.5 * torch.exp2(torch.randn((experts, 2, F.blocks(inner), F.blocks(hidden)), generator=g))).cuda()
    ds = (0.01 / inner ** 0.5 * torch.exp2(torch.randn((experts, F.blocks(hidden), F.blocks(inner)), generator=g))).cuda()
    return router, gu, gus, down, ds


def tokens_of(tokens, hidden, x_type, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((tokens, hidden), generator=g).to(x_type).cuda()


def call(x, lay, top_k, renormalize=True, y_type=None, pad=0, stream=None, workspace=None):
    router, gu, gus, down, ds = lay
    tokens, hidden = x.shape
    wide = torch.full((tokens + 1, hidden + pad), 7.0, dtype=y_type or x.dtype, device="cuda")
    ids, probs = torch.full((tokens, top_k), -1, dtype=torch.int32, device="cuda"), torch.full((tokens, top_k), -1.0, device="cuda")
    if workspace is None:
        workspace = torch.full((sqnn.sqnn_moe_workspace_bytes(tokens, top_k, gu.shape[2]),), 0xff, dtype=torch.uint8, device="cuda")
    sqnn.sqnn_moe_fp8(x, router, top_k, renormalize, gu, gus, down, ds, wide[:tokens, :hidden], workspace, ids, probs, stream)
    torch.cuda.synchronize()
    assert bool((wide[tokens] == 7).all()) and bool((wide[:tokens, hidden:] == 7).all())      # nothing beside the rows
    return wide[:tokens, :hidden], ids, probs


def check(x, lay, top_k, got, renormalize=True):
    router, gu, gus, down, ds = lay
    y, ids, probs = got
    tokens, hidden = x.shape
    inner = gu.shape[2]
    xd = x.double()
    logits = xd @ router.double().T
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), order.indices[:, :top_k])
    p = torch.softmax(order.values[:, :top_k] if renormalize else order.values, 1)[:, :top_k]
    exponent = 36 * EPS * (xd.abs() @ router.double().abs().T).amax(1, keepdim=True)
    assert bool(((probs.double() - p).abs() <= ((16 + 2 * top_k + router.shape[0] / 8) * EPS + exponent) * p + 1e-40).all())
    s_h, s_i = (158 + hidden / 64) * EPS, (158 + inner / 64) * EPS
    ref, tol = torch.zeros_like(xd), torch.zeros_like(xd)
    for e in torch.unique(ids).tolist():
        t, k = torch.nonzero(ids == e, as_tuple=True)
        wg, wu, wd = F.weight_values(gu[e, 0], gus[e, 0]), F.weight_values(gu[e, 1], gus[e, 1]), F.weight_values(down[e], ds[e])
        a, b = xd[t] @ wg.T, xd[t] @ wu.T
        da, db = s_h * (xd[t].abs() @ wg.abs().T), s_h * (xd[t].abs() @ wu.abs().T)
        silu = a * torch.sigmoid(a)
        v = silu * b
        dv = 1.1 * da * (b.abs() + db) + silu.abs() * db + 10 * EPS * v.abs()
        share = p[t, k][:, None]
        ref[t] += share * (v @ wd.T)
        tol[t] += share * (dv @ wd.abs().T + (s_i + (32 + 2 * top_k) * EPS + exponent[t]) * (v.abs() @ wd.abs().T))
    if y.dtype == BF16:
        tol = tol + F.HALF_STEP[BF16] * (ref.abs() + tol)
    off = (y.double() - ref).abs()
    assert bool((off <= tol + 1e-40).all()), float((off / (tol + 1e-40)).max())


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,experts,top_k", [(1, 1, 1), (1, 8, 2), (2, 5, 5), (5, 12, 3), (8, 64, 8), (9, 4, 2), (16, 100, 7), (33, 3, 2), (64, 6, 1), (64, 256, 16)])
@pytest.mark.parametrize("hidden,inner,x_type", [(1, 1, F32), (63, 17, BF16), (200, 130, F32), (256, 128, BF16), (1000, 500, F32)])
def test_sizes_and_types(tokens, experts, top_k, hidden, inner, x_type):
    lay, x = layer(experts, hidden, inner, x_type, tokens + hidden), tokens_of(tokens, hidden, x_type, hidden + experts)
    if hidden == 1:                                                # logits of one column are easily equal or opposite: keep them apart
        lay[0].copy_(torch.arange(1, experts + 1, device="cuda")[:, None])
    check(x, lay, top_k, call(x, lay, top_k, y_type=BF16 if tokens % 2 else F32, pad=tokens % 3))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,experts,top_k,hidden,inner", [(1, 64, 8, 2048, 1024), (16, 32, 4, 4096, 768), (3, 8, 2, 2000, 5000), (64, 16, 2, 1024, 1024)])
@pytest.mark.parametrize("x_type", [BF16, F32])
def test_larger(tokens, experts, top_k, hidden, inner, x_type):
    lay, x = layer(experts, hidden, inner, x_type, tokens), tokens_of(tokens, hidden, x_type, 5)
    for renormalize in (True, False):
        check(x, lay, top_k, call(x, lay, top_k, renormalize), renormalize)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,experts,top_k,hidden,inner,x_type", [
    (29, 8, 7, 367, 3264, F32), (2, 64, 8, 384, 2864, BF16), (3, 20, 4, 690, 1500, BF16), (5, 16, 6, 700, 2000, F32), (9, 12, 3, 1100, 2000, BF16),
    (64, 8, 4, 500, 3000, F32), (1, 9, 9, 17, 700, BF16)])
def test_rows_shared_by_a_cluster(tokens, experts, top_k, hidden, inner, x_type):
    lay, x = layer(experts, hidden, inner, x_type, tokens + inner), tokens_of(tokens, hidden, x_type, 10)
    first = call(x, lay, top_k)
    check(x, lay, top_k, first)
    assert all(torch.equal(a, b) for a, b in zip(call(x, lay, top_k), first))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,experts,top_k,hidden,inner,x_type", [
    (64, 8, 2, 3200, 400, BF16), (64, 8, 2, 4096, 384, F32), (20, 16, 3, 3300, 256, BF16), (25, 6, 6, 5000, 130, BF16),     # many tokens, wide outputs
    (32, 512, 16, 256, 128, BF16), (64, 256, 1, 128, 64, F32), (2, 512, 16, 300, 100, F32),                                # most experts, most logits
    (1, 2, 1, 11264, 300, F32), (3, 4, 2, 11264, 129, BF16), (5, 2, 2, 11264, 11264, F32), (64, 3, 3, 300, 11264, BF16)])  # widest
def test_limits(tokens, experts, top_k, hidden, inner, x_type):
    lay, x = layer(experts, hidden, inner, x_type, tokens + inner), tokens_of(tokens, hidden, x_type, 9)
    check(x, lay, top_k, call(x, lay, top_k))


@pytest.mark.gpu
def test_equal_logits_go_to_the_lowest_index():
    lay = layer(40, 96, 64, F32, 3)
    lay[0][:] = lay[0][0]                                          # all logits equal
    lay[0][30] *= 2
    x = tokens_of(4, 96, F32, 4).abs()
    lay[0].abs_()
    _, ids, probs = call(x, lay, 4)
    assert ids.tolist() == [[30, 0, 1, 2]] * 4
    check(x, lay, 4, call(x, lay, 4))


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
def test_strides_and_alignment(x_type):
    tokens, experts, hidden, inner = 6, 9, 250, 140
    lay, x = layer(experts, hidden, inner, x_type, 5), tokens_of(tokens, hidden, x_type, 6)
    want = call(x, lay, 3)
    router, gu, gus, down, ds = lay
    wide_x = torch.full((tokens, hidden + 5), float("nan"), dtype=x_type, device="cuda")
    wide_x[:, 1:hidden + 1] = x
    wide_r = torch.full((experts, hidden + 3), float("nan"), dtype=x_type, device="cuda")
    wide_r[:, 2:hidden + 2] = router
    wide_gu = torch.full((experts + 1, 3, inner + 2, 288), 0x7f, dtype=torch.uint8, device="cuda")     # NaN around the weights
    wide_gu[:experts, :2, :inner, :hidden] = gu.view(torch.uint8)
    wide_d = torch.full((experts, hidden + 1, 176), 0x7f, dtype=torch.uint8, device="cuda")
    wide_d[:, :hidden, :inner] = down.view(torch.uint8)
    moved = (wide_r[:, 2:hidden + 2], wide_gu.view(F.E4M3)[:experts, :2, :inner, :hidden], gus, wide_d.view(F.E4M3)[:, :hidden, :inner], ds)
    got = call(wide_x[:, 1:hidden + 1], moved, 3, pad=1)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    check(x, lay, 3, got)


@pytest.mark.gpu
def test_the_last_rows_may_end_with_their_data():
    # tensors that end with the last weight: a row's last 16 bytes are not all there
    experts, hidden, inner = 2, 50, 40
    lay, x = layer(experts, hidden, inner, F32, 7), tokens_of(3, hidden, F32, 8)
    router, gu, gus, down, ds = lay
    flat = torch.zeros(experts * 2 * inner * 64 - 14, dtype=torch.uint8, device="cuda").view(F.E4M3)
    tight = torch.as_strided(flat, (experts, 2, inner, hidden), (2 * inner * 64, inner * 64, 64, 1))
    tight.view(torch.uint8).copy_(gu.view(torch.uint8))
    check(x, lay, 2, call(x, (router, tight, gus, down, ds), 2))


@pytest.mark.gpu
def test_magnitudes_far_apart():
    lay, x = layer(6, 640, 256, F32, 9), tokens_of(4, 640, F32, 10)
    x[0] *= 1e-30
    x[1] *= 1e12
    x[2, ::7] *= 1e6
    x[3] = 0
    lay[0].mul_(1e-12)                                             # keeps the logits small
    lay[0][5] = 0
    lay[2][:, 1] *= 1e-8
    for top_k in (1, 6):
        got = call(x, lay, top_k)
        rows = [1, 2]
        check(x[rows], lay, top_k, tuple(t[rows] for t in got))
        assert bool((got[0][3] == 0).all()) and bool(torch.isfinite(got[0]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", [BF16, F32])
def test_not_finite(x_type):
    lay, x = layer(8, 300, 200, x_type, 11), tokens_of(12, 300, x_type, 12)
    x[3, 7] = float("nan")
    x[5, 8] = float("inf")
    y, ids, probs = call(x, lay, 2)
    assert bool(((ids >= 0) & (ids < 8)).all()) and bool((ids[:, 0] != ids[:, 1]).all())
    assert not bool(torch.isfinite(y[3]).any()) and not bool(torch.isfinite(y[5]).any())
    rest = [t for t in range(12) if t not in (3, 5)]
    check(x[rest], lay, 2, (y[rest], ids[rest], probs[rest]))      # other tokens do not notice


@pytest.mark.gpu
def test_results_are_the_same_from_run_to_run_and_whatever_the_workspace_holds():
    lay, x = layer(30, 700, 300, BF16, 13), tokens_of(20, 700, BF16, 14)
    first = call(x, lay, 4)
    n = sqnn.sqnn_moe_workspace_bytes(20, 4, 300)
    for fill in (0, 0xff, 0x3c):
        again = call(x, lay, 4, workspace=torch.full((n,), fill, dtype=torch.uint8, device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.gpu
def test_own_stream_graph_and_two_at_once():
    lay, a, b = layer(16, 512, 256, BF16, 15), tokens_of(4, 512, BF16, 16), tokens_of(13, 512, BF16, 17)
    want_a, want_b = call(a, lay, 2), call(b, lay, 2)
    router, gu, gus, down, ds = lay
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    ya, yb = torch.empty_like(a), torch.empty_like(b)
    wa, wb = (torch.empty(sqnn.sqnn_moe_workspace_bytes(t, 2, 256), dtype=torch.uint8, device="cuda") for t in (4, 13))
    torch.cuda.synchronize()
    for _ in range(10):
        sqnn.sqnn_moe_fp8(a, router, 2, True, gu, gus, down, ds, ya, wa, stream=s1)
        sqnn.sqnn_moe_fp8(b, router, 2, True, gu, gus, down, ds, yb, wb, stream=s2)
    torch.cuda.synchronize()
    assert torch.equal(ya, want_a[0]) and torch.equal(yb, want_b[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sqnn.sqnn_moe_fp8(a, router, 2, True, gu, gus, down, ds, ya, wa)
    a.copy_(tokens_of(4, 512, BF16, 18))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(ya, call(a, lay, 2)[0])


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,experts,hidden,inner", [(1, 4, 512, 256), (20, 8, 3500, 700), (3, 16, 400, 2500)])
def test_a_wait_that_gives_up_ends_the_call(tokens, experts, hidden, inner):
    lay, x = layer(experts, hidden, inner, F32, 21), tokens_of(tokens, hidden, F32, 22)
    good = call(x, lay, 2)
    router, gu, gus, down, ds = lay
    y, status = torch.zeros_like(x), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.zeros(sqnn.sqnn_moe_workspace_bytes(tokens, 2, inner), dtype=torch.uint8, device="cuda")
    sqnn.sqnn_set_debug_flags(16, 2_000_000)
    try:
        sqnn.sqnn_moe_fp8(x, router, 2, True, gu, gus, down, ds, y, ws, None, None, status)
        torch.cuda.synchronize()
    finally:
        sqnn.sqnn_set_debug_flags(0, 0)
    assert int(status.item()) == -sqnn.E_TIMEOUT
    assert bool((y == 0).all())
    assert all(torch.equal(a, b) for a, b in zip(call(x, lay, 2), good))       # the next call is not affected


@pytest.mark.gpu
def test_norm_then_layer():
    lay = layer(10, 768, 256, BF16, 19)
    g = torch.Generator().manual_seed(20)
    x, r, w = torch.randn((7, 768), generator=g), torch.randn((7, 768), generator=g).to(BF16), (torch.rand(768, generator=g) + 0.5).to(BF16)
    h, y = torch.empty((7, 768), dtype=BF16, device="cuda"), torch.empty((7, 768), dtype=BF16, device="cuda")
    sqnn.sqnn_rmsnorm_fp8(x.cuda(), w.cuda(), 1e-6, None, None, r.cuda(), h, y)
    got = call(y, lay, 3)
    assert bool(((y.cpu().double() - F.rmsnorm(x, w, 1e-6, r)[1]).abs() <= 2.0 ** -7 * y.cpu().double().abs()).all())
    check(y, lay, 3, got)


def c_layer(**changed):
    ok = dict(experts=8, top_k=2, hidden=256, inner=128, renormalize=1, reserved=0, router=4096, gate_up=4096, gate_up_scale=4096, down=4096, down_scale=4096,
              router_row=256, gate_up_expert=65536, gate_up_half=32768, gate_up_row=256, down_expert=32768, down_row=128)
    return sqnn.Moe(**{**ok, **changed})


def test_refusals_of_the_c_entry_point():
    f = sqnn.lib().sqnn_moe_fp8
    ok = dict(tokens=4, x=4096, xt=0, ldx=256, y=8192, yt=0, ldy=256, ids=None, probs=None, ws=65536, bytes=1 << 20)

    def rc(lay=None, **changed):
        return f(ctypes.byref(lay or c_layer()), *{**ok, **changed}.values(), None, None)

    assert f(None, *ok.values(), None, None) == sqnn.E_INVALID_ARG
    for bad in (dict(tokens=0), dict(x=None), dict(y=None), dict(xt=2), dict(yt=-1), dict(ldx=255), dict(ldy=255), dict(x=4098), dict(y=8193, yt=1), dict(ids=4097),
                dict(probs=4098)):
        assert rc(**bad) == sqnn.E_INVALID_ARG, bad
    for bad in (dict(experts=0), dict(top_k=0), dict(top_k=9), dict(hidden=0), dict(inner=0), dict(router=None), dict(gate_up=None), dict(gate_up_scale=None),
                dict(down=None), dict(down_scale=None), dict(router_row=255), dict(gate_up_row=240), dict(down_row=112), dict(gate_up_half=-16),
                dict(gate_up_expert=-16), dict(down_expert=-16), dict(gate_up_scale=4098), dict(down_scale=4097), dict(router=4097)):
        assert rc(c_layer(**bad)) == sqnn.E_INVALID_ARG, bad
    for bad in (dict(experts=513), dict(top_k=17, experts=32), dict(gate_up=4104), dict(down=4100), dict(gate_up_row=264), dict(down_row=136), dict(gate_up_half=32784), dict(gate_up_expert=65600), dict(down_expert=32784), dict(gate_up_expert=1 << 60), dict(gate_up_half=1 << 60),
                dict(down_expert=1 << 60),
                dict(hidden=(1 << 20) + 1, router_row=1 << 21, gate_up_row=1 << 21), dict(inner=(1 << 20) + 1, down_row=1 << 21)):
        lay = c_layer(**bad)
        assert rc(lay, ldx=1 << 21, ldy=1 << 21) == sqnn.E_UNSUPPORTED, bad
    assert rc(tokens=65) == sqnn.E_UNSUPPORTED
    assert rc(c_layer(experts=300), tokens=64) == sqnn.E_UNSUPPORTED
    need = sqnn.sqnn_moe_workspace_bytes(4, 2, 128)
    assert need > 0 and sqnn.sqnn_moe_workspace_bytes(65, 2, 128) == 0 and sqnn.sqnn_moe_workspace_bytes(4, 2, 11265) == 0
    for bad in (dict(ws=None), dict(bytes=need - 1), dict(ws=65536 + 128)):
        assert rc(**bad) == sqnn.E_WORKSPACE, bad


@pytest.mark.gpu
def test_refusals_of_the_binding():
    lay, x = layer(4, 256, 128, F32, 1), tokens_of(2, 256, F32, 1)
    router, gu, gus, down, ds = lay
    good = dict(d_x=x, d_router=router, top_k=2, renormalize=True, d_gate_up=gu, d_gate_up_scale=gus, d_down=down, d_down_scale=ds, d_y=torch.empty_like(x),
                d_workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    sqnn.sqnn_moe_fp8(**good)
    for bad in (dict(d_x=x.cpu()), dict(d_router=router.bfloat16()), dict(d_router=router[:, :255]), dict(d_gate_up=gu[:3]), dict(d_gate_up=gu.view(torch.uint8)),
                dict(d_gate_up=gu[:, :1]), dict(d_down=down[:, :255]), dict(d_down_scale=ds[:, :1]), dict(d_gate_up_scale=gus.double()), dict(d_y=x[:1]),
                dict(d_ids=torch.empty((2, 2), device="cuda")), dict(d_probs=torch.empty((2, 1), device="cuda")), dict(d_y=x.half()), dict(d_down=None),
                dict(d_ids=torch.empty((2, 2), dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            sqnn.sqnn_moe_fp8(**{**good, **bad})
    for bad, status in ((dict(d_workspace=None), sqnn.E_WORKSPACE), (dict(d_workspace=good["d_workspace"][:100]), sqnn.E_WORKSPACE),
                        (dict(top_k=5), sqnn.E_INVALID_ARG), (dict(top_k=0), sqnn.E_INVALID_ARG)):
        with pytest.raises(sqnn.SqnnError) as e:
            sqnn.sqnn_moe_fp8(**{**good, **bad})
        assert e.value.status == status
