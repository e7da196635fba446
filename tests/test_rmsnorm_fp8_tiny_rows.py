"""``sqnn_rmsnorm_fp8`` on rows so small that 1 / rms is no fp32 number's power of two: every scale and 8-bit number is still the definition's, those of
groups of zeros among them."""
import pytest
import torch

from tests import fp8_helpers as F
from tests.test_rmsnorm_fp8 import call, check

F32, BF16 = F.F32, F.BF16


@pytest.mark.gpu
@pytest.mark.parametrize("n", [300, 1024, 20000])
@pytest.mark.parametrize("x_type,residual,weight", [(F32, None, F32), (F32, F32, BF16), (BF16, None, BF16), (BF16, BF16, F32)])
def test_a_group_of_zeros_in_a_row_of_tiny_values(n, x_type, residual, weight):
    g = torch.Generator().manual_seed(n)
    magnitudes = torch.tensor([1e-37, 1e-38, 1e-39, 4e-40, 1e-42, 2.0 ** -148])
    x = (torch.randn((6, n), generator=g).sign() * (1 + torch.rand((6, n), generator=g)) * magnitudes[:, None]).to(x_type)
    x[:, 0] = 2.0 ** -133                                          # (the smallest bf16 number: a row of zeros would be another case)
    x[:, 128:256] = 0
    w = (torch.rand(n, generator=g) + 0.5).to(weight)
    r = None if residual is None else torch.zeros((6, n)).to(residual)
    for eps in (0.0, 1e-300):
        got = call(x, w, eps, r, F32)
        assert bool((got[2].float()[:, 128:256] == 0).all())
        check(x, w, eps, r, got, F32)


@pytest.mark.gpu
@pytest.mark.parametrize("weight", [F32, BF16])
def test_small_weights_on_a_row_of_tiny_values(weight):
    g = torch.Generator().manual_seed(5)
    x = torch.randn((3, 640), generator=g).sign() * torch.tensor([1e-40, 1e-43, 2.0 ** -149])[:, None]
    w = torch.rand(640, generator=g) + 0.5
    w[128:256] *= 2.0 ** -98                                       # y stays above 2^-100 there
    w[256:384] *= 2.0 ** 60
    w = w.to(weight)
    check(x, w, 0.0, None, call(x, w, 0.0))
