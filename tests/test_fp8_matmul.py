"""``sqnn_fp8_matmul`` against the sum of the definition in 64 bits.

Tolerance of an output, in units of A = sum_c |W X| (in 64 bits).  Products of two e4m3 numbers are exact in fp32.  The roundings: a block's
128 products are added up by four MMA instructions into an fp32 accumulator.  An instruction adds 32 products and the accumulator, aligned to
the largest; with at least 25 bits kept per addend (what the fp32 result has, and one) that is at most 33 units of 2^-24 of
the block's magnitudes per instruction, 132 for the four.  The product of two scales and the addition of a scaled block are two roundings, and the additions of a block to the
running sum one each, kblocks in all, split sums eight more: (132 + 2 + kblocks + 8) 2^-24 A.  bf16 output: half a step of the value more."""
import pytest
import torch

from paper_1905_10138_b200 import sqnn
from tests import fp8_helpers as F

F32, BF16 = F.F32, F.BF16


def operands(m, n, batch, seed, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    w, x = F.random_fp8((m, n), g, device), F.random_fp8((batch, n), g, device)
    ws = torch.exp2(torch.randn((F.blocks(m), F.blocks(n)), generator=g) * 2).to(device)
    xs = torch.exp2(torch.randn((batch, F.blocks(n)), generator=g) * 2).to(device)
    return w, ws, x, xs


def expected(w, ws, x, xs):
    wv, xv = F.weight_values(w, ws), F.activation_values(x, xs)
    return xv @ wv.T, xv.abs() @ wv.abs().T


def product(w, ws, x, xs, y_type=F32, pad=0, stream=None):
    batch, m = x.shape[0], w.shape[0]
    wide = torch.full((batch + 1, m + pad), 77.0, dtype=y_type, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sqnn.sqnn_fp8_matmul(w, ws, x, xs, wide[:batch, :m], status, stream)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert bool((wide[batch] == 77).all()) and bool((wide[:batch, m:] == 77).all())      # nothing beside the rows
    return wide[:batch, :m]


def run(m, n, batch, y_type=F32, pad=0, seed=1):
    ops = operands(m, n, batch, seed)
    y = product(*ops, y_type, pad)
    ref, total = expected(*ops)
    tol = (142 + F.blocks(n)) * 2.0 ** -24 * total + 1e-40
    if y_type == BF16:
        tol = tol + F.HALF_STEP[BF16] * (ref.abs() + tol)
    off = (y.double() - ref).abs()
    assert bool((off <= tol).all()), (float((off / total.clamp(min=1e-30)).max()), float((off / tol).max()))
    return ops, y


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 2, 8, 15, 16, 17, 31, 33, 64, 65, 100, 128, 129, 257, 500])
@pytest.mark.parametrize("m,n", [(1, 1), (5, 17), (127, 128), (128, 129), (130, 1000), (1000, 2050), (300, 4500)])
def test_sizes(m, n, batch):
    run(m, n, batch, F32 if (m + batch) % 2 else BF16, pad=(m + n) % 3)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,batch", [(4096, 9216, 1), (6000, 3000, 8), (4096, 9216, 64), (4096, 4096, 512), (2000, 700, 3000), (8192, 256, 1100), (129, 16384, 130),
                                       (20000, 130, 70), (40000, 200, 3), (256, 40000, 20)])
@pytest.mark.parametrize("y_type", [F32, BF16])
def test_larger(m, n, batch, y_type):
    run(m, n, batch, y_type)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,batch", [(4099, 300, 1500), (1030, 4000, 1025), (700, 900, 129), (1500, 2000, 4200)])
@pytest.mark.parametrize("y_type", [F32, BF16])
@pytest.mark.parametrize("pad", [0, 1, 2, 4])
def test_rows_of_y_on_and_off_boundaries(m, n, batch, y_type, pad):
    run(m, n, batch, y_type, pad)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [3, 40, 200])
def test_strides(batch):
    ops = operands(260, 900, batch, 4)
    spread = []
    for t in ops:                                                  # rows 32 or 5 elements further apart, the gaps NaN
        bits = t.view(torch.uint8) if t.element_size() == 1 else t
        wide = torch.full((t.shape[0], -(-t.shape[1] // 16) * 16 + 32 if t.element_size() == 1 else t.shape[1] + 5),
                          0x7f if t.element_size() == 1 else float("nan"), dtype=bits.dtype, device="cuda")
        wide[:, :t.shape[1]] = bits
        spread.append((wide.view(t.dtype) if t.element_size() == 1 else wide)[:, :t.shape[1]])
    assert torch.equal(product(*ops), product(*spread, pad=3))


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 48, 130, 300, 4000])
def test_results_are_the_same_from_run_to_run(batch):
    ops = operands(1030, 5000, batch, 5)
    first = product(*ops)
    for _ in range(5):
        assert torch.equal(first, product(*ops))


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [2, 70])
def test_not_finite(batch):
    w, ws, x, xs = operands(300, 400, batch, 6)
    w.view(torch.uint8)[7, 300] = 0x7f                             # NaN: its row of W, in all of Y
    x.view(torch.uint8)[1, 5] = 0xff                               # its row of Y
    ws[1, 0] = float("inf")                                        # rows 128 .. 255: infinity times whatever sums there
    y = product(w, ws, x, xs)
    nan = torch.isnan(y)
    assert bool(nan[1].all()) and bool(nan[:, 7].all())
    fine = torch.ones((batch, 300), dtype=torch.bool, device="cuda")
    fine[1] = fine[:, 7] = fine[:, 128:256] = False
    assert not bool(nan[fine].any())
    assert not bool(torch.isfinite(y[:, 128:256]).any())


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [4, 90])
def test_zero_scales_and_extremes(batch):
    w, ws, x, xs = operands(200, 300, batch, 7)
    xs[0] = 0.0
    xs[1] = 2.0 ** -126
    ws[0, 1] = 2.0 ** 60
    y = product(w, ws, x, xs)
    ref, total = expected(w, ws, x, xs)
    off = (y.double() - ref).abs()
    assert bool((off <= 150 * 2.0 ** -24 * total + 1e-40).all())
    assert bool((y[0] == 0).all())


@pytest.mark.gpu
def test_own_stream_graph_and_two_at_once():
    a, b = operands(1000, 2000, 5, 8), operands(512, 4096, 300, 9)
    ya, yb = product(*a), product(*b)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [(torch.empty_like(ya), torch.empty_like(yb)) for _ in range(8)]
    torch.cuda.synchronize()
    for oa, ob in outs:
        sqnn.sqnn_fp8_matmul(*a, oa, None, s1)
        sqnn.sqnn_fp8_matmul(*b, ob, None, s2)
    torch.cuda.synchronize()
    assert all(torch.equal(oa, ya) and torch.equal(ob, yb) for oa, ob in outs)
    g, out = torch.cuda.CUDAGraph(), torch.zeros_like(ya)
    with torch.cuda.graph(g):
        sqnn.sqnn_fp8_matmul(*a, out)
    a[2].view(torch.uint8).copy_(operands(1000, 2000, 5, 10)[2].view(torch.uint8))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, product(*a))


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,batch,y_type,pad", [(2560, 256, 2048, F32, 0), (2430, 700, 2020, BF16, 3), (2305, 1300, 1793, F32, 1), (256, 130, 19200, BF16, 0),
                                                  (8192, 300, 1200, BF16, 8), (300, 2000, 9601, F32, 0)])
def test_tiles_of_a_last_round(m, n, batch, y_type, pad):
    run(m, n, batch, y_type, pad)


@pytest.mark.gpu
def test_all_forms_at_once_on_streams_of_their_own():
    """Clusters of several kernels share SMs and their tensor memory."""
    sizes = [(1000, 6000, 3), (900, 5000, 30), (700, 9000, 60), (500, 7000, 100), (1024, 4000, 700), (8192, 512, 1500)]
    ops = [operands(*size, 20 + i) for i, size in enumerate(sizes)]
    want, streams = [product(*o) for o in ops], [torch.cuda.Stream() for _ in ops]
    outs = [[torch.empty_like(y) for y in want] for _ in range(12)]
    torch.cuda.synchronize()
    for row in outs:
        for o, y, s in zip(ops, row, streams):
            sqnn.sqnn_fp8_matmul(*o, y, None, s)
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for row in outs for y, w in zip(row, want))


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,batch", [(300, 4000, 7), (300, 4000, 90), (4096, 300, 2000), (4096, 4000, 500)])
def test_a_wait_that_gives_up_ends_the_call(m, n, batch):
    ops = operands(m, n, batch, 11)
    good = product(*ops)
    y, status = torch.zeros_like(good), torch.zeros(1, dtype=torch.int32, device="cuda")
    sqnn.sqnn_set_debug_flags(8, 2_000_000)
    try:
        sqnn.sqnn_fp8_matmul(*ops, y, status)
        torch.cuda.synchronize()
    finally:
        sqnn.sqnn_set_debug_flags(0, 0)
    assert int(status.item()) == -sqnn.E_TIMEOUT
    assert torch.equal(product(*ops), good)                        # the next call is not affected


@pytest.mark.gpu
def test_norm_then_product():
    g = torch.Generator().manual_seed(12)
    x, r = torch.randn((20, 1000), generator=g), torch.randn((20, 1000), generator=g).to(BF16)
    weight = torch.rand(1000, generator=g) + 0.5
    w, ws, _, _ = operands(700, 1000, 1, 13)
    d_h, q, s = torch.empty((20, 1000), dtype=BF16, device="cuda"), F.rows16((20, 1000), "cuda"), torch.empty((20, 8), device="cuda")
    sqnn.sqnn_rmsnorm_fp8(x.cuda(), weight.cuda(), 1e-6, q, s, r.cuda(), d_h)
    y = product(w, ws, q, s)
    _, _, qe, se = F.rmsnorm(x, weight, 1e-6, r)
    xv = qe.cuda() * se.double().repeat_interleave(128, 1)[:, :1000].cuda()
    wv = F.weight_values(w, ws)
    off = (y.double() - xv @ wv.T).abs()
    assert bool((off <= 150 * 2.0 ** -24 * (xv.abs() @ wv.abs().T)).all())


def test_refusals_of_the_c_entry_point():
    f = sqnn.lib().sqnn_fp8_matmul
    ok = dict(m=256, n=300, batch=4, w=4096, ldw=304, ws=8192, ldws=3, x=16384, ldx=304, xs=32768, ldxs=3, y=65536, yt=0, ldy=256)

    def rc(**changed):
        return f(*{**ok, **changed}.values(), None, None)

    for bad in (dict(m=0), dict(n=0), dict(batch=0), dict(w=None), dict(ws=None), dict(x=None), dict(xs=None), dict(y=None), dict(yt=2), dict(ldw=288),
                dict(ldx=288), dict(ldws=2), dict(ldxs=2), dict(ldy=255), dict(ws=8193), dict(xs=32770), dict(y=65538), dict(y=65537, yt=1)):
        assert rc(**bad) == sqnn.E_INVALID_ARG, bad
    for bad in (dict(w=4097), dict(x=16392), dict(ldw=305), dict(ldx=312), dict(m=(1 << 30) + 1, ldy=1 << 31), dict(batch=(1 << 30) + 1)):
        assert rc(**bad) == sqnn.E_UNSUPPORTED, bad


def test_refusals_of_the_binding():
    w, ws, x, xs = operands(10, 20, 2, 1, "cpu")
    y = torch.zeros((2, 10))
    with pytest.raises(ValueError, match="current CUDA device"):
        sqnn.sqnn_fp8_matmul(w, ws, x, xs, y)
    with pytest.raises(ValueError):
        sqnn.sqnn_fp8_matmul(w, None, x, xs, y)


@pytest.mark.gpu
def test_refusals_of_the_binding_on_the_device():
    w, ws, x, xs = operands(256, 300, 2, 1)
    good = dict(d_w=w, d_w_scale=ws, d_x=x, d_x_scale=xs, d_y=torch.zeros((2, 256), device="cuda"))
    for bad in (dict(d_w=w.view(torch.uint8)), dict(d_x=x.view(torch.uint8)), dict(d_w=w[:, :299]), dict(d_w_scale=ws[:1]), dict(d_x_scale=xs[:, :2]),
                dict(d_y=good["d_y"][:, :255]), dict(d_y=good["d_y"].half()), dict(d_x=x[0]), dict(d_w_scale=ws.double()), dict(d_x_scale=xs.cpu()),
                dict(d_status=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            sqnn.sqnn_fp8_matmul(**{**good, **bad})
    shifted = torch.zeros((2, 320), dtype=torch.uint8, device="cuda").view(F.E4M3)[:, 8:308]
    with pytest.raises(sqnn.SqnnError) as e:
        sqnn.sqnn_fp8_matmul(**{**good, "d_x": shifted})
    assert e.value.status == sqnn.E_UNSUPPORTED
