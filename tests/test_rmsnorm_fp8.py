"""``sqnn_rmsnorm_fp8`` against its definition in 64 bits.  h, scale and q are compared number for number: the call promises
what exact arithmetic gives.  y in fp32 has four roundings (h 2^k w, 1 / rms to 32 bits, their product, and the 64-bit steps that round
to less than one), in bf16 one more."""
import pytest
import torch

from paper_1905_10138_b200 import sqnn
from tests import fp8_helpers as F

F32, BF16, E4M3 = F.F32, F.BF16, F.E4M3


def inputs(batch, n, x, residual, weight, seed):
    g = torch.Generator().manual_seed(seed)
    xs = torch.randn((batch, n), generator=g)
    xs[:, torch.randint(0, n, (max(1, n // 100),), generator=g)] *= 30
    r = None if residual is None else (2 * torch.randn((batch, n), generator=g)).to(residual)
    return xs.to(x), r, (1 + 0.2 * torch.randn(n, generator=g)).to(weight)


def call(x, w, eps, residual=None, y=None, want_q=True, q=None, pad=0, shift=0, stream=None):
    """Runs the call on copies of CPU tensors on the GPU, with rows `pad` elements further apart and `shift` elements off a boundary."""
    def place(t):
        if t is None:
            return None
        wide = torch.full((t.shape[0], t.shape[1] + pad + shift), 7.0, dtype=t.dtype, device="cuda")
        view = wide[:, shift:shift + t.shape[1]]
        view.copy_(t)
        return view
    batch, n = x.shape
    d_x, d_r = place(x), place(residual)
    d_h = None if residual is None else place(torch.full_like(residual, 3.0))
    d_q = None
    if want_q:
        wide = torch.full((batch, n + pad + shift), 0x55, dtype=torch.uint8, device="cuda")
        d_q = wide.view(E4M3)[:, shift:shift + n]
    d_s = torch.full((batch, F.blocks(n)), 5.0, device="cuda") if want_q else None
    d_y = None if y is None else place(torch.full((batch, n), 9.0, dtype=y))
    sqnn.sqnn_rmsnorm_fp8(d_x, w.cuda(), eps, d_q, d_s, d_r, d_h, d_y, stream)
    torch.cuda.synchronize()
    if want_q and pad + shift:
        assert bool((wide[:, :shift] == 0x55).all()) and bool((wide[:, shift + n:] == 0x55).all())      # nothing beside the rows
    return tuple(None if t is None else t.cpu() for t in (d_h, d_y, d_q, d_s))


def same(a, b):
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    a, b = torch.nan_to_num(a.double(), nan=0.25), torch.nan_to_num(b.double(), nan=0.25)
    assert torch.equal(a, b), f"{int((a != b).sum())} of {a.numel()} differ"


def check(x, w, eps, residual, got, y_type=None):
    h, y, q, scale = F.rmsnorm(x, w, eps, residual)
    if residual is not None:
        same(got[0], h)
    if y_type is not None:
        tol = 4 * 2.0 ** -24 + (F.HALF_STEP[BF16] if y_type == BF16 else 0)
        off = (got[1].double() - y).abs()
        assert bool((off <= tol * y.abs() + 1e-40).all()), float((off / y.abs().clamp(min=1e-30)).max())
    if got[2] is not None:
        same(got[3], scale)
        same(got[2].float(), q)


@pytest.mark.gpu
@pytest.mark.parametrize("batch,n", [(1, 1), (2, 7), (3, 127), (5, 128), (4, 129), (333, 3001), (70, 4096), (9, 8197), (3, 16384), (2, 16385), (2, 40000)])
@pytest.mark.parametrize("x,residual,weight,y", [(BF16, BF16, BF16, None), (F32, None, F32, F32), (F32, BF16, BF16, BF16), (BF16, F32, F32, None),
                                                 (BF16, None, BF16, BF16), (F32, F32, BF16, F32)])
def test_sizes_and_types(batch, n, x, residual, weight, y):
    xs, r, w = inputs(batch, n, x, residual, weight, 10 * n + batch)
    check(xs, w, 1e-5, r, call(xs, w, 1e-5, r, y), y)


@pytest.mark.gpu
@pytest.mark.parametrize("pad,shift", [(8, 0), (16, 0), (5, 0), (3, 1), (8, 8)])
@pytest.mark.parametrize("n", [200, 1024, 16500])
def test_strides_and_alignment(n, pad, shift):
    xs, r, w = inputs(6, n, BF16, BF16, BF16, n + pad)
    check(xs, w, 1e-6, r, call(xs, w, 1e-6, r, BF16, pad=pad, shift=shift), BF16)


@pytest.mark.gpu
def test_values_on_the_border_between_two_numbers():
    # every middle between two neighbours and the largest number: y / scale is rstd / fl(rstd) off the middle, on either side
    codes = torch.arange(127, dtype=torch.uint8).view(E4M3).double()
    middle = (codes[1:] + codes[:-1]) / 2
    rows = []
    for k in range(64):
        v = torch.cat([middle * (-1) ** k, torch.tensor([448.0, 0.0])])
        rows.append(v * 2.0 ** (k % 20 - 10))
    x = torch.stack(rows).float()
    x[:, 125] *= torch.linspace(0.5, 0.9, 64)                      # rows differ in their norm
    for eps in (0.0, 1e-3):
        check(x, torch.ones(128), eps, None, call(x, torch.ones(128), eps, None, F32), F32)
    b = (x / 2).to(BF16)
    check(b, torch.ones(128, dtype=BF16), 1e-6, None, call(b, torch.ones(128, dtype=BF16), 1e-6))


@pytest.mark.gpu
def test_sum_lands_on_a_middle_of_bf16():
    # fp32 + bf16 whose fp32 sum lies on a middle between two bf16 numbers although the exact sum does not
    r = torch.tensor([[1.0, 1.0, -1.0, 1.0, 2.0 ** 10, 1.0]]).to(BF16)
    x = torch.tensor([[2.0 ** -8 + 2.0 ** -32, 2.0 ** -8 - 2.0 ** -32, -2.0 ** -8 - 2.0 ** -32, 3 * 2.0 ** -8 - 2.0 ** -31, 4 + 2.0 ** -20, 2.0 ** -8]])
    w = torch.ones(6)
    check(x, w, 1e-6, r, call(x, w, 1e-6, r, F32), F32)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [300, 20000])
def test_rows_of_zeros_of_extremes_and_not_finite(n):
    xs, _, w = inputs(8, n, F32, None, F32, 3)
    xs[0] = 0
    xs[1] *= 1e-36
    xs[2] *= 1e34
    xs[3, 5] = float("inf")
    xs[4, 6] = float("nan")
    xs[5, 7] = float("-inf")
    xs[6, 128:256] = 0                                             # a group of zeros inside a row
    xs[7] = torch.finfo(F32).min
    for eps in (1e-6, 0.0):
        got = call(xs, w, eps)
        check(xs, w, eps, None, got)


@pytest.mark.gpu
def test_in_place_and_only_y():
    xs, r, w = inputs(5, 777, BF16, BF16, BF16, 8)
    d_x, d_r, d_w = xs.cuda(), r.cuda(), w.cuda()
    q, s = F.rows16((5, 777), "cuda"), torch.empty((5, 7), device="cuda")
    sqnn.sqnn_rmsnorm_fp8(d_x, d_w, 1e-6, q, s, d_r, d_r, d_x)     # h over the residual, y over x
    check(xs, w, 1e-6, r, (d_r.cpu(), d_x.cpu(), q.cpu(), s.cpu()), BF16)
    check(xs, w, 1e-6, r, call(xs, w, 1e-6, r, F32, want_q=False), F32)


@pytest.mark.gpu
def test_own_stream_and_graph_replay():
    xs, r, w = inputs(17, 1000, F32, BF16, BF16, 4)
    d_x, d_r, d_w = xs.cuda(), r.cuda(), w.cuda()
    h, q, s = torch.empty_like(d_r), F.rows16((17, 1000), "cuda"), torch.empty((17, 8), device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        sqnn.sqnn_rmsnorm_fp8(d_x, d_w, 1e-6, q, s, d_r, h)
    stream.synchronize()
    check(xs, w, 1e-6, r, (h.cpu(), None, q.cpu(), s.cpu()))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sqnn.sqnn_rmsnorm_fp8(d_x, d_w, 1e-6, q, s, d_r, h)
    other, r2, _ = inputs(17, 1000, F32, BF16, BF16, 5)
    d_x.copy_(other)
    d_r.copy_(r2)
    g.replay()
    torch.cuda.synchronize()
    check(other, w, 1e-6, r2, (h.cpu(), None, q.cpu(), s.cpu()))


def test_refusals_of_the_c_entry_point():
    f, ok = sqnn.lib().sqnn_rmsnorm_fp8, dict(batch=2, n=256, x=4096, xt=0, ldx=256, r=None, rt=0, ldr=0, h=None, ldh=0, w=8192, wt=0, eps=1e-6, q=16384,
                                              ldq=256, s=32768, lds=2, y=None, yt=0, ldy=0)

    def rc(**changed):
        return f(*{**ok, **changed}.values(), None)

    bad = [dict(batch=0), dict(n=0), dict(x=None), dict(w=None), dict(q=None, s=None), dict(q=None), dict(s=None), dict(xt=7), dict(wt=-1), dict(ldx=255),
           dict(ldq=255), dict(lds=1), dict(r=4096, ldr=256), dict(h=4096, ldh=256), dict(r=4096, ldr=255, h=4096, ldh=256),
           dict(r=4096, ldr=256, h=4096, ldh=255), dict(r=4096, ldr=256, h=4096, ldh=256, rt=3), dict(y=4096, ldy=255), dict(y=4096, ldy=256, yt=2),
           dict(eps=-1e-6), dict(eps=float("nan")), dict(x=4098), dict(w=8193), dict(s=32770), dict(y=4097, ldy=256, yt=1)]
    for b in bad:
        assert rc(**b) == sqnn.E_INVALID_ARG, b
    assert rc(n=(1 << 30) + 1, ldx=1 << 31, ldq=1 << 31, lds=1 << 31) == sqnn.E_UNSUPPORTED
    assert rc(batch=1 << 31) == sqnn.E_UNSUPPORTED


def test_refusals_of_the_binding():
    x, w = torch.zeros((2, 256)), torch.zeros(256)
    q, s = F.rows16((2, 256)), torch.zeros((2, 2))
    with pytest.raises(ValueError, match="current CUDA device"):
        sqnn.sqnn_rmsnorm_fp8(x, w, 1e-6, q, s)
    with pytest.raises(TypeError):
        sqnn.sqnn_rmsnorm_fp8(x.numpy(), w, 1e-6, q, s)
    with pytest.raises(ValueError):
        sqnn.sqnn_rmsnorm_fp8(None, w, 1e-6, q, s)


@pytest.mark.gpu
def test_refusals_of_the_binding_on_the_device():
    x, w = torch.zeros((2, 256), device="cuda"), torch.zeros(256, device="cuda")
    q, s = F.rows16((2, 256), "cuda"), torch.zeros((2, 2), device="cuda")
    good = dict(d_x=x, d_weight=w, eps=1e-6, d_q=q, d_scale=s)
    for bad in (dict(d_x=x.half()), dict(d_x=x[0]), dict(d_x=x.t()), dict(d_weight=w[:255]), dict(d_weight=w.half()), dict(d_q=q.view(torch.uint8)),
                dict(d_q=q[:1]), dict(d_scale=s[:, :1]), dict(d_scale=s.double()), dict(d_h=x), dict(d_residual=x, d_h=x.bfloat16()),
                dict(d_y=x.half()), dict(d_y=x[:, :255]), dict(d_residual=x[:1], d_h=x), dict(d_weight=w.cpu())):
        with pytest.raises(ValueError):
            sqnn.sqnn_rmsnorm_fp8(**{**good, **bad})
    for bad in (dict(d_q=None), dict(d_scale=None), dict(d_residual=x), dict(d_q=None, d_scale=None), dict(d_x=x[:1].expand(2, 256))):
        with pytest.raises(sqnn.SqnnError) as e:
            sqnn.sqnn_rmsnorm_fp8(**{**good, **bad})
        assert e.value.status == sqnn.E_INVALID_ARG
