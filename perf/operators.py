"""Performance cases of the 8-bit serving operators: the calls a user of them makes, with their sizes.

Three operators, each through the public Python entry points:

- ``product``: ``sqnn_fp8_matmul``, a layer whose weights are kept in 8-bit floating point with a scale for each
  128 x 128 block, times activations with a scale for each 128 columns of a row;
- ``norm``: ``sqnn_rmsnorm_fp8``, the residual's addition, the root-mean-square norm and the conversion to 8 bits with
  scales, which is what stands before such a product;
- ``moe``: ``sqnn_moe_fp8``, a mixture-of-experts layer of such weights for a few tokens, router included.

``own`` selects between their plain form in elementary torch operations and the framework's kernels.
"""
import torch

own = False

BLOCK = 128
TOP = 448.0                      # largest number of 8 bits with four exponent bits
EPS = 1e-6


def _product(name, m, n, batch, y):
    c = {"op": "product", "m": m, "n": n, "batch": batch, "y": y}
    return dict(c, name=name) if name else c


def _norm(name, batch, n, x, residual, y):
    c = {"op": "norm", "batch": batch, "n": n, "x": x, "residual": residual, "y": y}
    return dict(c, name=name) if name else c


def _moe(name, tokens, experts, top_k, hidden, inner, x):
    c = {"op": "moe", "tokens": tokens, "experts": experts, "top_k": top_k, "hidden": hidden, "inner": inner, "x": x}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a small layer, one token: launch and latency
        _product("product_small_b1", 1024, 1024, 1, "bf16"),
        # AlexNet FC6 kept in 8 bits, one activation vector
        _product("product_fc6_b1", 4096, 9216, 1, "f32"),
        # the gates of an LSTM, rows that are no multiple of the block, eight requests at once
        _product("product_lstm_b8", 6000, 3000, 8, "bf16"),
        # AlexNet FC6 over a batch
        _product("product_fc6_b64", 4096, 9216, 64, "f32"),
        # a transformer's feed-forward matrix, a prompt of 512 tokens
        _product("product_ffn_b512", 4096, 16384, 512, "bf16"),
        # the same matrix, a batch of prompts: bound by the tensor cores
        _product("product_ffn_b4096", 4096, 16384, 4096, "bf16"),
        # before a product, one token
        _norm("norm_b1", 1, 4096, "bf16", "bf16", "none"),
        # odd sizes; the fp32 output of a product joins a bf16 residual, the norm also wanted as bf16
        _norm("norm_odd_b333", 333, 3001, "f32", "bf16", "bf16"),
        # a batch of prompts
        _norm("norm_b8192", 8192, 4096, "bf16", "bf16", "none"),
        # one token, many small experts
        _moe("moe_t1_e64", 1, 64, 8, 2048, 1024, "bf16"),
        # odd sizes and few experts, fp32 activations
        _moe("moe_odd_t5_e12", 5, 12, 3, 1000, 500, "f32"),
        # a decoding batch that reaches most experts
        _moe("moe_t16_e64", 16, 64, 8, 4096, 1536, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _size(rng, lo, hi):
    """Most sizes are multiples of a power of two."""
    v, step = _log(rng, lo, hi), rng.choice((1, 8, 64, 128))
    return max(lo, v // step * step)


def draw(rng):
    """A call of any size between the smallest and the largest listed ones of its operator."""
    op = rng.choice(("product", "product", "norm", "moe"))
    if op == "product":
        m, n = _size(rng, 100, 8192), _size(rng, 100, 16384)
        batch = min(_log(rng, 1, 4096), max(1, (1 << 38) // (m * n)))
        return _product("", m, n, batch, rng.choice(("f32", "bf16")))
    if op == "norm":
        n = _size(rng, 64, 16384)
        batch = min(_log(rng, 1, 16384), (1 << 25) // n)
        return _norm("", batch, n, rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16", "none")), rng.choice(("none", "none", "f32", "bf16")))
    experts = rng.choice((6, 8, 16, 32, 60, 64, 128))
    top_k = rng.randint(1, min(8, experts))
    hidden = _size(rng, 256, 4096)
    inner = min(_size(rng, 128, 4096), max(128, (1 << 30) // (3 * experts * hidden)))
    return _moe("", _log(rng, 1, 32), experts, top_k, hidden, inner, rng.choice(("bf16", "bf16", "f32")))


def _type(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _rows16(shape):
    """An uninitialised 8-bit tensor whose rows start on 16-byte boundaries."""
    padded = -(-shape[-1] // 16) * 16
    return torch.zeros((*shape[:-1], padded), dtype=torch.float8_e4m3fn, device="cuda")[..., :shape[-1]]


def _blocks(n):
    return -(-n // BLOCK)


def _quantized_matrix(w):
    """An fp32 matrix in 8 bits with a scale for each 128 x 128 block, as such weights are stored."""
    m, n = w.shape
    full = torch.zeros((_blocks(m) * BLOCK, _blocks(n) * BLOCK), device="cuda")
    full[:m, :n] = w
    b = full.view(_blocks(m), BLOCK, _blocks(n), BLOCK)
    scale = b.abs().amax((1, 3)).clamp(min=1e-30) / TOP
    q = _rows16((m, n))
    q.copy_((b / scale[:, None, :, None]).view(full.shape)[:m, :n])
    return q, scale


def _quantized_rows(x):
    """fp32 activations in 8 bits with a scale for each row and 128 columns."""
    batch, n = x.shape
    full = torch.zeros((batch, _blocks(n) * BLOCK), device="cuda")
    full[:, :n] = x
    b = full.view(batch, _blocks(n), BLOCK)
    scale = b.abs().amax(2).clamp(min=1e-30) / TOP
    q = _rows16((batch, n))
    q.copy_((b / scale[:, :, None]).view(full.shape)[:, :n])
    return q, scale


def _activations(shape, g):
    """Normal values, some columns far larger than the rest, as the residual stream of a model has them."""
    x = torch.randn(shape, device="cuda", generator=g)
    x[:, torch.randint(0, shape[1], (max(1, shape[1] // 200),), device="cuda", generator=g)] *= 20
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    if case["op"] == "product":
        m, n, batch = case["m"], case["n"], case["batch"]
        s["w"], s["w_scale"] = _quantized_matrix(torch.randn((m, n), device="cuda", generator=g) * 0.02)
        s["x"], s["x_scale"] = _quantized_rows(_activations((batch, n), g))
        s["out"] = torch.empty((batch, m), dtype=_type(case["y"]), device="cuda")
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    elif case["op"] == "norm":
        batch, n = case["batch"], case["n"]
        s["in"] = _activations((batch, n), g).to(_type(case["x"]))
        s["weight"] = (1 + 0.1 * torch.randn(n, device="cuda", generator=g)).to(_type(case["x"]))
        s["res"] = s["h"] = s["out"] = None
        if case["residual"] != "none":
            s["res"] = (3 * _activations((batch, n), g)).to(_type(case["residual"]))
            s["h"] = torch.empty_like(s["res"])
        s["q"] = _rows16((batch, n))
        s["scale"] = torch.empty((batch, _blocks(n)), device="cuda")
        if case["y"] != "none":
            s["out"] = torch.empty((batch, n), dtype=_type(case["y"]), device="cuda")
    else:
        tokens, experts, top_k, hidden, inner = (case[k] for k in ("tokens", "experts", "top_k", "hidden", "inner"))
        s["in"] = torch.randn((tokens, hidden), device="cuda", generator=g).to(_type(case["x"]))
        s["router"] = (torch.randn((experts, hidden), device="cuda", generator=g) * 2 / hidden ** 0.5).to(_type(case["x"]))
        s["gate_up"], s["down"] = _rows16((experts, 2, inner, hidden)), _rows16((experts, hidden, inner))
        s["gate_up_scale"] = torch.empty((experts, 2, _blocks(inner), _blocks(hidden)), device="cuda")
        s["down_scale"] = torch.empty((experts, _blocks(hidden), _blocks(inner)), device="cuda")
        for e in range(experts):
            for k in range(2):
                q, scale = _quantized_matrix(torch.randn((inner, hidden), device="cuda", generator=g) / hidden ** 0.5)
                s["gate_up"][e, k].copy_(q)
                s["gate_up_scale"][e, k] = scale
            q, scale = _quantized_matrix(torch.randn((hidden, inner), device="cuda", generator=g) / inner ** 0.5)
            s["down"][e].copy_(q)
            s["down_scale"][e] = scale
        s["out"] = torch.empty((tokens, hidden), dtype=_type(case["x"]), device="cuda")
        s["ids"] = torch.empty((tokens, top_k), dtype=torch.int32, device="cuda")
        s["probs"] = torch.empty((tokens, top_k), device="cuda")
        s["workspace"] = torch.empty(65536 + 8 * tokens * top_k * (inner + 128), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms

def _spread(scale, rows, cols):
    """Scales of 128 x 128 blocks as a matrix of rows x cols."""
    return scale.repeat_interleave(BLOCK, -2)[..., :rows, :].repeat_interleave(BLOCK, -1)[..., :cols]


def _weights(q, scale):
    return q.float() * _spread(scale, q.shape[-2], q.shape[-1])


def _round_to(v, dtype):
    """64-bit numbers rounded once (torch goes through 32 bits)."""
    f = v.float()
    if dtype == torch.float32:
        return f
    off = v - f.double()
    up, down = torch.full_like(f, torch.inf), torch.full_like(f, -torch.inf)
    border = (f.view(torch.int32) & 0xffff) == 0x8000
    f = torch.where(border & (off > 0), torch.nextafter(f, up), torch.where(border & (off < 0), torch.nextafter(f, down), f))
    return f.to(dtype)


def _round_fp8(v):
    """64-bit numbers of at most 448 rounded once to 8 bits: three bits behind the leading one, steps of 2^-9 at least."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def _plain_product(s):
    x = s["x"].float() * s["x_scale"].repeat_interleave(BLOCK, 1)[:, :s["n"]]
    return (x @ _weights(s["w"], s["w_scale"]).T).to(s["out"].dtype)


def _plain_norm(s):
    # 64 bits: which 8-bit number a value rounds to is decided at a border
    h, n = s["in"].double(), s["n"]
    got = {}
    if s["res"] is not None:
        got["h"] = _round_to(h + s["res"].double(), s["res"].dtype)
        h = got["h"].double()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].double()
    b = torch.nn.functional.pad(y, (0, -n % BLOCK)).view(s["batch"], -1, BLOCK)
    got["scale"] = (b.abs().amax(2) / TOP).float().clamp(min=2.0 ** -126)
    got["q"] = _round_fp8((b / got["scale"].double()[:, :, None]).view(s["batch"], -1)[:, :n]).to(torch.float8_e4m3fn)
    if s["out"] is not None:
        got["y"] = _round_to(y, s["out"].dtype)
    return got


def _plain_moe(s):
    # logits in 64 bits: which experts are taken is decided at a border
    probs = torch.softmax(s["in"].double() @ s["router"].double().T, 1)
    probs, ids = torch.sort(probs, dim=1, descending=True, stable=True)
    probs, ids = probs[:, :s["top_k"]], ids[:, :s["top_k"]]
    probs = (probs / probs.sum(1, keepdim=True)).float()
    x = s["in"].float()
    if s["tokens"] * s["top_k"] < s["experts"]:                        # the chosen experts' weights, one by one
        pick = ids.flatten()
        x = x.repeat_interleave(s["top_k"], 0)[:, :, None]
        gate = (_weights(s["gate_up"][pick, 0], s["gate_up_scale"][pick, 0]) @ x)[:, :, 0]
        up = (_weights(s["gate_up"][pick, 1], s["gate_up_scale"][pick, 1]) @ x)[:, :, 0]
        inner = gate / (1 + torch.exp(-gate)) * up
        y = (_weights(s["down"][pick], s["down_scale"][pick]) @ inner[:, :, None])[:, :, 0]
        y = (y.view(s["tokens"], s["top_k"], -1) * probs[:, :, None]).sum(1)
    else:                                                              # all experts for all tokens
        gate = x @ _weights(s["gate_up"][:, 0], s["gate_up_scale"][:, 0]).transpose(1, 2)
        up = x @ _weights(s["gate_up"][:, 1], s["gate_up_scale"][:, 1]).transpose(1, 2)
        inner = gate / (1 + torch.exp(-gate)) * up
        share = torch.zeros((s["tokens"], s["experts"]), device="cuda").scatter_(1, ids, probs)
        y = ((inner * share.T[:, :, None]) @ _weights(s["down"], s["down_scale"]).transpose(1, 2)).sum(0)
    return {"y": y.to(s["out"].dtype), "ids": ids.int(), "probs": probs}


def run(state):
    s = state
    if own:
        from paper_1905_10138_b200 import sqnn
        if s["op"] == "product":
            sqnn.sqnn_fp8_matmul(s["w"], s["w_scale"], s["x"], s["x_scale"], s["out"], s["status"])
            return s["out"]
        if s["op"] == "norm":
            sqnn.sqnn_rmsnorm_fp8(s["in"], s["weight"], EPS, s["q"], s["scale"], s["res"], s["h"], s["out"])
            got = {"scale": s["scale"], "q": s["q"]}
            if s["h"] is not None:
                got["h"] = s["h"]
            if s["out"] is not None:
                got["y"] = s["out"]
            return got
        sqnn.sqnn_moe_fp8(s["in"], s["router"], s["top_k"], True, s["gate_up"], s["gate_up_scale"], s["down"], s["down_scale"],
                          s["out"], s["workspace"], s["ids"], s["probs"])
        return {"y": s["out"], "ids": s["ids"], "probs": s["probs"]}
    return {"product": _plain_product, "norm": _plain_norm, "moe": _plain_moe}[s["op"]](s)


def work(case):
    if case["op"] == "product":
        m, n, batch = case["m"], case["n"], case["batch"]
        scales = 4 * _blocks(n) * (_blocks(m) + batch)
        return {"bytes": m * n + batch * n + scales + batch * m * (4 if case["y"] == "f32" else 2), "flops": 2 * m * n * batch}
    if case["op"] == "norm":
        size = {"f32": 4, "bf16": 2, "none": 0}
        batch, n = case["batch"], case["n"]
        per = size[case["x"]] + 2 * size[case["residual"]] + size[case["y"]] + 1
        return {"bytes": batch * n * per + n * size[case["x"]] + 4 * batch * _blocks(n), "flops": 8 * batch * n}
    tokens, experts, top_k, hidden, inner = (case[k] for k in ("tokens", "experts", "top_k", "hidden", "inner"))
    reached = experts * (1 - (1 - top_k / experts) ** tokens)          # experts that some token takes, on average
    size = 4 if case["x"] == "f32" else 2
    scales = 4 * 3 * _blocks(hidden) * _blocks(inner)
    return {"bytes": reached * (3 * hidden * inner + scales) + size * hidden * (experts + 2 * tokens) + 8 * tokens * top_k,
            "flops": 6 * tokens * top_k * hidden * inner + 2 * tokens * experts * hidden}


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _exact_weights(q, scale):
    rows = torch.arange(q.shape[0], device="cuda") // BLOCK
    cols = torch.arange(q.shape[1], device="cuda") // BLOCK
    return q.double() * scale.double()[rows][:, cols]


def _exact_fp8(v):
    """Each value's nearest 8-bit number, ties to the even one, by search among all of them."""
    codes = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    middle = (codes[1:] + codes[:-1]) / 2
    a = v.abs()
    low, high = torch.searchsorted(middle, a, right=False), torch.searchsorted(middle, a, right=True)
    at = torch.where(low == high, low, torch.where(low % 2 == 0, low, high))     # on a middle: the even code
    return codes[at] * torch.sign(v)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "product":
        cols = torch.arange(case["n"], device="cuda") // BLOCK
        return (s["x"].double() * s["x_scale"].double()[:, cols]) @ _exact_weights(s["w"], s["w_scale"]).T
    if case["op"] == "norm":
        got, h, n = {}, s["in"].double(), case["n"]
        if s["res"] is not None:
            h = h + s["res"].double()
            if s["res"].dtype == torch.bfloat16:                       # eight bits, ties to even
                _, e = torch.frexp(h)
                step = torch.ldexp(torch.ones_like(h), e - 8)
                h = torch.round(h / step) * step
            else:
                h = h.float().double()
            got["h"] = h
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / n + EPS) * s["weight"].double()
        groups = torch.arange(n, device="cuda") // BLOCK
        most = torch.zeros((case["batch"], _blocks(n)), dtype=torch.float64, device="cuda")
        most.scatter_reduce_(1, groups.expand(case["batch"], n), y.abs(), "amax")
        scale = (most / TOP).float().double().clamp(min=2.0 ** -126)   # the scale is an fp32 number by definition
        got["scale"] = scale
        got["q"] = _exact_fp8(y / scale[:, groups])
        if s["out"] is not None:
            got["y"] = y
        return got
    x = s["in"].double()
    logits = x @ s["router"].double().T
    y = torch.zeros((case["tokens"], case["hidden"]), dtype=torch.float64, device="cuda")
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    ids = order.indices[:, :case["top_k"]]
    top = torch.exp(order.values[:, :case["top_k"]] - order.values[:, :1])
    probs = top / top.sum(1, keepdim=True)
    for e in torch.unique(ids).tolist():
        t, k = torch.nonzero(ids == e, as_tuple=True)
        gate = x[t] @ _exact_weights(s["gate_up"][e, 0], s["gate_up_scale"][e, 0]).T
        up = x[t] @ _exact_weights(s["gate_up"][e, 1], s["gate_up_scale"][e, 1]).T
        inner = gate * torch.sigmoid(gate) * up
        y[t] += probs[t, k][:, None] * (inner @ _exact_weights(s["down"][e], s["down_scale"][e]).T)
    return {"y": y, "ids": ids.int(), "probs": probs}
