"""Workloads of the 8-bit floating-point operators: norm, quantizer and linear layers with scales for blocks of 128.

Each case names one operator, its sizes and types.  ``prepare`` makes what a serving program holds before the call,
``run`` is one pass through the operator: in its plain form (elementary torch operations in 32 bits, rounded once at
the end), or, with ``own`` set, through this package.  ``exact`` gives the same outputs from the definition in 64 bits.

    norm      h = x + residual; y = h / sqrt(mean(h^2) + eps) * gain; y as e4m3 codes with one scale for each row and
              128 columns, or in the inputs' type, or both; h in the inputs' type
    quantize  v = x, or silu(gate) * x; v as e4m3 codes with one scale for each row and 128 columns
    linear    y = x W^T + b; x as the two above write it, W in e4m3 codes with one scale for each 128 x 128 block
"""
import math

import torch

own = False

BLOCK = 128
TOP = 448.0                   # largest e4m3 value
MIN_SCALE = 2.0 ** -100       # scale of a block of zeros
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
F8 = torch.float8_e4m3fn


# ---- cases ------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of one request between two layers: launch latency is everything
        dict(name="norm-1x2048", op="norm", rows=1, k=2048, residual=True, codes=True, values=False, dtype="bf16"),
        # the verified tokens of a few requests, a width that fills no block; 16-bit values for the layers that stay in 16 bits
        dict(name="norm-37x10001", op="norm", rows=37, k=10001, residual=True, codes=True, values=True, dtype="f16"),
        # the first norm of a long prompt
        dict(name="norm-16384x8192", op="norm", rows=16384, k=8192, residual=True, codes=True, values=False, dtype="bf16"),
        # attention's output of a decoding batch, on its way into the output projection
        dict(name="quantize-64x4096", op="quantize", rows=64, k=4096, gate=False, dtype="bf16"),
        # gated activation of a batch of tokens, odd sizes
        dict(name="gate-509x5003", op="quantize", rows=509, k=5003, gate=True, dtype="f16"),
        # gated activation of a long prompt, gate and value as halves of one projection's output
        dict(name="gate-8192x28672", op="quantize", rows=8192, k=28672, gate=True, dtype="bf16"),
        # the 1000-way classifier on 1024 features, one image or token: latency
        dict(name="linear-1x1024-1000", op="linear", rows=1, n=1000, k=1024, bias=True, dtype="f16"),
        # one token through a wide layer: a pure stream of weights, larger than the L2 cache
        dict(name="linear-1x8192-28672", op="linear", rows=1, n=28672, k=8192, bias=False, dtype="bf16"),
        # a decoding batch, sizes that fill no tile: ragged rows, columns and last block
        dict(name="linear-45x10001-5003", op="linear", rows=45, n=5003, k=10001, bias=True, dtype="f16"),
        # a large decoding batch: weights and products both count
        dict(name="linear-256x8192-10240", op="linear", rows=256, n=10240, k=8192, bias=False, dtype="bf16"),
        # prompts of odd lengths together through a mid-size layer
        dict(name="linear-1777x4096-6144", op="linear", rows=1777, n=6144, k=4096, bias=False, dtype="bf16"),
        # a long prompt through the widest layer: the tensor cores' rate
        dict(name="linear-8192x8192-28672", op="linear", rows=8192, n=28672, k=8192, bias=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(["norm", "quantize", "linear", "linear"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    k = _log(rng, 250, 12000)
    k = k if rng.random() < 0.4 else max(256, k // 256 * 256)               # widths are multiples more often than not
    rows = _log(rng, 1, 8192)
    if op == "norm":
        codes = rng.random() < 0.8
        return dict(op=op, rows=rows, k=k, residual=rng.random() < 0.7, codes=codes, values=not codes or rng.random() < 0.3,
                    dtype=rng.choice([dtype, dtype, dtype, "f32"]))
    if op == "quantize":
        return dict(op=op, rows=rows, k=k, gate=rng.random() < 0.6, dtype=dtype)
    n = _log(rng, 250, 28672)
    n = n if rng.random() < 0.4 else max(256, n // 256 * 256)
    return dict(op=op, rows=min(rows, 8192 * 8192 * 28672 // (n * k)), n=n, k=k, bias=rng.random() < 0.4, dtype=dtype)


# ---- inputs ------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _channels(g, x, strength):
    """A few channels that are stronger than the others, as activations have them."""
    k = x.shape[-1]
    x[:, torch.randint(0, k, (max(1, k // 200),), generator=g, device="cuda")] *= strength
    return x


def _pitched(x, multiple=8):
    """The same rows, each starting on a multiple of that many elements."""
    rows, k = x.shape
    wide = x.new_empty(rows, -(-k // multiple) * multiple)
    wide[:, :k] = x
    return wide[:, :k]


def _pad_blocks(x):
    """[rows][blocks][128], zeros behind a short last block."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK)).unflatten(1, (-1, BLOCK))


def _blocks(v):
    """e4m3 codes of v [rows][k] with the scale of each row's 128 columns."""
    cut = _pad_blocks(v)
    scales = (cut.abs().amax(2) / TOP).clamp(min=MIN_SCALE)
    return (cut / scales[..., None]).flatten(1)[:, :v.shape[1]].to(F8), scales


def _norm_inputs(case, seed):
    g, t = _gen(seed), TYPES[case["dtype"]]
    rows, k = case["rows"], case["k"]
    x = _pitched(_channels(g, _randn(g, rows, k), 6.0).to(t))
    residual = _pitched(_channels(g, _randn(g, rows, k) * 3.0, 20.0).to(t)) if case["residual"] else None
    return dict(x=x, residual=residual, gain=(1.0 + 0.2 * _randn(g, k)).to(t), eps=1e-5)


def _quantize_inputs(case, seed):
    """Gate and value lie beside each other, as one projection writes them."""
    g, t = _gen(seed), TYPES[case["dtype"]]
    rows, k = case["rows"], case["k"]
    pitch = -(-k // 8) * 8
    both = _channels(g, _randn(g, rows, 2 * pitch), 5.0).to(t)
    return dict(gate=both[:, :k] if case["gate"] else None, x=both[:, pitch:pitch + k])


def _linear_inputs(case, seed):
    g, t = _gen(seed), TYPES[case["dtype"]]
    rows, n, k = case["rows"], case["n"], case["k"]
    codes, scales = _blocks(_channels(g, _randn(g, rows, k), 8.0))
    w = _randn(g, n, k).mul_(100.0).clamp_(-TOP, TOP).to(F8)
    w_scales = (0.5 + torch.rand(-(-n // BLOCK), -(-k // BLOCK), generator=g, device="cuda")) / (100.0 * math.sqrt(k))
    bias = (_randn(g, n) * 0.1).to(t) if case["bias"] else None
    return dict(codes=_pitched(codes, 16), scales=scales, w=w, w_scales=w_scales, bias=bias)


_INPUTS = {"norm": _norm_inputs, "quantize": _quantize_inputs, "linear": _linear_inputs}
_handle = None


def prepare(case, seed):
    """What a serving program has in hand: the inputs and, for this package, the handle and the plan that it keeps."""
    global _handle
    state = _INPUTS[case["op"]](case, seed)
    state["case"] = case
    if own:
        from paper_1806_08342_b200 import qtz
        if _handle is None:
            _handle = qtz.Handle(0)
        state["handle"] = _handle
        if case["op"] == "linear":
            state["plan"] = _handle.f8_linear_create(state["w"], state["w_scales"], bias=state["bias"])
    return state


# ---- one pass ----------------------------------------------------------------------------------------------
def run(state):
    return _RUN[state["case"]["op"]](state)


def _given(**outputs):
    return {name: v for name, v in outputs.items() if v is not None}


def _norm(s):
    case = s["case"]
    if own:
        codes, scales, values, total = s["handle"].f8_rmsnorm(s["x"], s["gain"], s["eps"], residual=s["residual"], codes=case["codes"],
                                                              values=case["values"])
        return _given(codes=codes, scales=scales, values=values, sum=total)
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + s["eps"]) * s["gain"].float()
    codes, scales = _blocks(y) if case["codes"] else (None, None)
    t = s["x"].dtype
    return _given(codes=codes, scales=scales, values=y.to(t) if case["values"] else None, sum=h.to(t) if s["residual"] is not None else None)


def _quantize(s):
    if own:
        codes, scales = s["handle"].f8_quantize(s["x"], gate=s["gate"])
        return dict(codes=codes, scales=scales)
    v = s["x"].float()
    if s["gate"] is not None:
        g = s["gate"].float()
        v = v * (g / (1.0 + torch.exp(-g)))
    codes, scales = _blocks(v)
    return dict(codes=codes, scales=scales)


def _linear(s):
    if own:
        return s["plan"](s["codes"], s["scales"], dtype=TYPES[s["case"]["dtype"]])
    case = s["case"]
    n, k = case["n"], case["k"]
    column, row = torch.arange(k, device="cuda") // BLOCK, torch.arange(n, device="cuda") // BLOCK
    x = s["codes"].float() * s["scales"][:, column]
    w = s["w"].float() * s["w_scales"][row][:, column]
    y = torch.matmul(x, w.t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(TYPES[case["dtype"]])


_RUN = {"norm": _norm, "quantize": _quantize, "linear": _linear}


# ---- what a pass cannot do without ---------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    rows, k = case["rows"], case["k"]
    blocks = -(-k // BLOCK)
    coded = rows * (k + 4 * blocks)
    if case["op"] == "norm":
        return {"bytes": rows * k * size * (1 + 2 * case["residual"] + case["values"]) + k * size + coded * case["codes"], "flops": 6 * rows * k}
    if case["op"] == "quantize":
        return {"bytes": rows * k * size * (1 + case["gate"]) + coded, "flops": (8 if case["gate"] else 3) * rows * k}
    n = case["n"]
    return {"bytes": n * k + 4 * blocks * -(-n // BLOCK) + coded + size * rows * n + (size * n if case["bias"] else 0), "flops": 2 * rows * n * k}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------
def exact(case, seed):
    return _EXACT[case["op"]](case, _INPUTS[case["op"]](case, seed))


def _exact_codes(v):
    """What the codes stand for before they are rounded, and the scales, one block of columns after the other."""
    codes, scales = torch.empty_like(v), []
    for at in range(0, v.shape[1], BLOCK):
        cut = v[:, at:at + BLOCK]
        s = torch.clamp(torch.max(torch.abs(cut), dim=1).values / 448, min=2.0 ** -100)
        codes[:, at:at + BLOCK] = cut / s[:, None]
        scales.append(s)
    return codes, torch.stack(scales, 1)


def _exact_norm(case, s):
    h = s["x"].double() if s["residual"] is None else s["x"].double() + s["residual"].double()
    length = torch.sqrt(torch.sum(h ** 2, dim=1) / case["k"] + s["eps"])
    y = h / length[:, None] * s["gain"].double()
    out = {}
    if case["codes"]:
        out["codes"], out["scales"] = _exact_codes(y)
    if case["values"]:
        out["values"] = y
    if s["residual"] is not None:
        out["sum"] = h
    return out


def _exact_quantize(case, s):
    v = s["x"].double()
    if s["gate"] is not None:
        v *= s["gate"].double() * torch.sigmoid(s["gate"].double())
    codes, scales = _exact_codes(v)
    return dict(codes=codes, scales=scales)


def _exact_linear(case, s):
    rows, n, k = case["rows"], case["n"], case["k"]
    total = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
    each = torch.arange(n, device="cuda") // BLOCK
    for j, at in enumerate(range(0, k, BLOCK)):
        x = s["codes"][:, at:at + BLOCK].double() * s["scales"][:, j:j + 1].double()
        w = s["w"][:, at:at + BLOCK].double() * s["w_scales"][:, j].double()[each][:, None]
        total.addmm_(x, w.t())
    return total if s["bias"] is None else total + s["bias"].double()


_EXACT = {"norm": _exact_norm, "quantize": _exact_quantize, "linear": _exact_linear}
