"""What the tests of the 8-bit operators share: the number format and the definitions in 64 bits, on the CPU."""
import torch

BLOCK = 128
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}      # a rounding is off by at most this, relative to the value


def blocks(n):
    return -(-n // BLOCK)


def rows16(shape, device="cpu"):
    """A zeroed 8-bit tensor whose rows start on 16-byte boundaries."""
    padded = -(-shape[-1] // 16) * 16
    return torch.zeros((*shape[:-1], padded), dtype=torch.uint8, device=device).view(E4M3)[..., :shape[-1]]


def round_fp8(v):
    """64-bit numbers rounded once to e4m3 (nearest, ties to even), as 64-bit numbers."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).clamp(-448, 448)


def round_bf16(v):
    """64-bit numbers rounded once to bf16, as 64-bit numbers."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 8).clamp(min=-133))
    return torch.where(torch.isfinite(v), torch.round(v / step) * step, v)


def rmsnorm(x, weight, eps, residual=None):
    """(h, y, q, scale) in 64 bits from CPU tensors."""
    h = x.double()
    if residual is not None:
        h = h + residual.double()
        h = round_bf16(h) if residual.dtype == BF16 else h.float().double()
    n = h.shape[1]
    y = h * (1 / torch.sqrt((h * h).sum(1, keepdim=True) / n + eps)) * weight.double()
    g = torch.nn.functional.pad(y, (0, -n % BLOCK)).view(h.shape[0], -1, BLOCK)
    scale = (g.abs().amax(2) / 448).float().clamp(min=2.0 ** -126)
    q = round_fp8((g / scale.double()[:, :, None]).view(h.shape[0], -1)[:, :n])
    return h, y, q, scale


def weight_values(q, scale):
    """Weights of a matrix with a scale per 128 x 128 block, in 64 bits."""
    m, n = q.shape
    s = scale.double().repeat_interleave(BLOCK, 0)[:m].repeat_interleave(BLOCK, 1)[:, :n]
    return q.float().double() * s


def activation_values(q, scale):
    return q.float().double() * scale.double().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def random_fp8(shape, g, device="cpu"):
    """Numbers of all magnitudes e4m3 has, both signs, zeros among them, no NaN; rows on 16-byte boundaries."""
    q = rows16(shape, device)
    codes = torch.randint(0, 127, shape, generator=g, dtype=torch.uint8) | (torch.randint(0, 2, shape, generator=g, dtype=torch.uint8) << 7)
    q.view(torch.uint8).copy_(codes)
    return q
