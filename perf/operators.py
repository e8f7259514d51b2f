"""Workloads of the serving operators: 4-bit linear layers and the 8-bit key/value cache.

Each case names one operator, its sizes and types.  ``prepare`` makes what a decoding program holds before the
call, ``run`` is one pass through the operator: in its plain form (elementary torch operations in 32 bits,
rounded once at the end), or, with ``own`` set, through this package.  ``exact`` gives the same outputs from the
definition in 64 bits.

    linear     y = x W^T + b; W holds 4-bit codes with a scale (and optionally a zero point) per row and group
               of columns
    schedule   from the lengths of the requests: new blocks from the free list into the block tables, the slot of
               every new token, the row starts of the requests and their lengths after the step
    append     new keys and values quantized into the paged 8-bit cache, one scale per block and head; then the
               values that the touched blocks now stand for are read back
    attention  softmax attention of the new tokens over the paged 8-bit cache, causal by position, grouped heads
"""
import math
import random

import torch

own = False

MIN_SCALE = 2.0 ** -100
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases ------------------------------------------------------------------------------------------------
def listed():
    return [
        # the 1000-way classifier on 1024 features, one image or token: launch latency is everything
        dict(name="linear-1x1024-1000", op="linear", rows=1, n=1000, k=1024, group=32, zeros=False, bias=True, dtype="f16"),
        # one token through a wide layer with zero points: a pure stream of weights, larger than the L2 cache
        dict(name="linear-1x8192-32768", op="linear", rows=1, n=32768, k=8192, group=128, zeros=True, bias=False, dtype="bf16"),
        # a dozen requests, sizes that fill no tile: ragged rows, columns and last group
        dict(name="linear-12x10001-5003", op="linear", rows=12, n=5003, k=10001, group=64, zeros=False, bias=True, dtype="f16"),
        # a decoding batch through the widest layer
        dict(name="linear-32x8192-28672", op="linear", rows=32, n=28672, k=8192, group=128, zeros=False, bias=False, dtype="bf16"),
        # a decoding step of a mid-size server: one token each
        dict(name="schedule-decode-96", op="schedule", requests=96, new_min=1, new_max=1, cached_max=4000, block=32, width=160, lens=1),
        # an admission step: many requests, prompts beside decoding ones and idle ones
        dict(name="schedule-prompts-1501", op="schedule", requests=1501, new_min=0, new_max=83, cached_max=2000, block=16, width=160, lens=2),
        # one new token for each of 192 requests
        dict(name="append-decode-192", op="append", requests=192, new_min=1, new_max=1, cached_max=2000, heads=8, dim=128, block=32, dtype="bf16", lens=3),
        # prompts of odd lengths written at once
        dict(name="append-prompts-23", op="append", requests=23, new_min=17, new_max=1700, cached_max=50, heads=8, dim=128, block=64, dtype="bf16", lens=4),
        # one short conversation on a small model: latency
        dict(name="attention-1x77", op="attention", requests=1, len_min=77, len_max=77, new=1, kv_heads=4, group=4, dim=64, block=16, window=0, dtype="f16", lens=5),
        # four drafted tokens to verify for each of 16 requests, sliding window
        dict(name="attention-verify-16", op="attention", requests=16, len_min=301, len_max=6000, new=5, kv_heads=8, group=3, dim=128, block=16, window=1024, dtype="bf16", lens=6),
        # one request over a very long document: the work has to be split along the cache
        dict(name="attention-1x262143", op="attention", requests=1, len_min=262143, len_max=262143, new=1, kv_heads=4, group=8, dim=128, block=64, window=0, dtype="bf16", lens=7),
        # a full decoding batch, lengths over two orders of magnitude
        dict(name="attention-64x32768", op="attention", requests=64, len_min=300, len_max=32768, new=1, kv_heads=8, group=4, dim=128, block=32, window=0, dtype="bf16", lens=8),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(["linear", "schedule", "append", "attention"])
    dtype = rng.choice(["bf16", "f16"])
    if op == "linear":
        return dict(op=op, rows=_log(rng, 1, 32), n=_log(rng, 250, 28672), k=_log(rng, 250, 8192), group=rng.choice([32, 64, 128]),
                    zeros=rng.random() < 0.5, bias=rng.random() < 0.5, dtype=dtype)
    if op == "schedule":
        block, cached = rng.choice([16, 32, 64]), _log(rng, 30, 4000)
        new_min, new_max = rng.choice([(1, 1), (0, 5), (0, 83)])
        return dict(op=op, requests=_log(rng, 1, 1501), new_min=new_min, new_max=new_max, cached_max=cached, block=block,
                    width=-(-(cached + new_max) // block) + rng.randrange(3), lens=rng.randrange(1 << 20))
    if op == "append":
        new_min, new_max = rng.choice([(1, 1), (1, 9), (17, _log(rng, 20, 1700))])
        return dict(op=op, requests=_log(rng, 1, 192 if new_max < 10 else 23), new_min=new_min, new_max=new_max, cached_max=_log(rng, 10, 2000),
                    heads=rng.choice([1, 2, 4, 8]), dim=rng.choice([64, 128, 256]), block=rng.choice([16, 32, 64, 128]), dtype=dtype,
                    lens=rng.randrange(1 << 20))
    kv_heads, dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 256])
    requests = _log(rng, 1, 64)
    top = min(262143, (64 * 32768 * 8 * 128) // (requests * kv_heads * dim))
    len_max = _log(rng, 20, top)
    return dict(op=op, requests=requests, len_min=max(8, len_max // rng.choice([1, 2, 50])), len_max=len_max, new=rng.choice([1, 1, 1, 2, 5, 8]),
                kv_heads=kv_heads, group=rng.choice([1, 2, 3, 4, 8]), dim=dim, block=rng.choice([16, 32, 64, 128]),
                window=rng.choice([0, 0, 0, 200, 1024]), dtype=dtype, lens=rng.randrange(1 << 20))


# ---- lengths: part of the case, so that its work is known ------------------------------------------------------
def _spread(case, lo, hi, salt):
    """Whole numbers over [lo, hi], spread over their logarithm where that spans more than a factor of ten."""
    rng = random.Random(case["lens"] * 7 + salt)
    if hi > 10 * max(lo, 1):
        return [min(hi, max(lo, int(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi + 1)))) - (lo == 0 and rng.random() < 0.1))) for _ in range(case["requests"])]
    return [rng.randint(lo, hi) for _ in range(case["requests"])]


def _step_lengths(case):
    """(tokens cached, tokens new) of every request of a schedule or append case."""
    return _spread(case, 0, case["cached_max"], 1), _spread(case, case["new_min"], case["new_max"], 2)


def _cache_lengths(case):
    """Tokens in the cache of every request of an attention case, its new ones included; the longest is there once."""
    got = _spread(case, case["len_min"], case["len_max"], 3)
    got[0] = case["len_max"]
    return [max(v, case["new"]) for v in got]


# ---- inputs ------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _linear_inputs(case, seed):
    """Activations with a few strong channels, codes of normal weights, scales that differ from group to group."""
    g, t = _gen(seed), TYPES[case["dtype"]]
    rows, n, k = case["rows"], case["n"], case["k"]
    groups = -(-k // case["group"])
    pitch = -(-k // 8) * 8                                   # rows of activations start on 16 bytes
    x = _randn(g, rows, pitch)
    x[:, torch.randint(0, k, (max(1, k // 200),), generator=g, device="cuda")] *= 8.0
    x = x.to(t)[:, :k]
    codes = torch.empty(n, (k + 1) // 2, dtype=torch.uint8, device="cuda")
    zeros = torch.randint(5, 11, (n, groups), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    for half in range(2):                                    # element 2i in the low nibble, 2i + 1 in the high one
        q = torch.clamp(torch.round(_randn(g, *codes.shape) * 2.6), -8, 7).to(torch.int8)
        q = (q + 8 if zeros is not None else q & 15).to(torch.uint8)
        codes = q if half == 0 else codes | (q << 4)
    if k % 2:
        codes[:, -1] &= 15
    scales = ((0.5 + torch.rand(n, groups, generator=g, device="cuda")) / (2.6 * math.sqrt(k))).to(t)
    bias = (_randn(g, n) * 0.1).to(t) if case["bias"] else None
    return dict(x=x, codes=codes, scales=scales, zeros=zeros, bias=bias)


def _schedule_inputs(case, seed):
    """Block tables that hold the cached tokens, ids in the order a long-running server leaves them in."""
    cached, new = _step_lengths(case)
    block, width = case["block"], case["width"]
    have = [-(-c // block) for c in cached]
    need = sum(-(-(c + m) // block) - h for c, m, h in zip(cached, new, have))
    pool = sum(have) + need + 100
    ids = torch.randperm(pool, generator=_gen(seed), device="cuda").to(torch.int32)
    have_t, at = _ints(have), torch.arange(width, device="cuda")
    first = torch.cumsum(have_t, 0) - have_t
    table = torch.where(at[None] < have_t[:, None], ids[(first[:, None] + at[None]).clamp(max=pool - 1)], -1).to(torch.int32).contiguous()
    free = ids[sum(have):].contiguous()
    return dict(cached=_ints(cached), new=_ints(new), table=table, free=free, free_count=_ints([free.numel()]), capacity=sum(new) + 7)


def _codes(g, *shape):
    return torch.clamp(torch.round(_randn(g, *shape).mul_(40.0)), -127, 127).to(torch.int8)


def _append_inputs(case, seed):
    """Keys and values as slices of one projection's output; blocks that are partly filled already."""
    g, t = _gen(seed), TYPES[case["dtype"]]
    cached, new = _step_lengths(case)
    heads, dim, block = case["heads"], case["dim"], case["block"]
    # only the blocks that the step touches are in this pool: the first holds the request's last cached tokens
    counts = [-(-(c + m) // block) - c // block for c, m in zip(cached, new)]
    blocks = sum(counts) + 3
    ids = torch.randperm(blocks, generator=g, device="cuda")
    slots, touched, first = [], [], 0
    for c, m, n in zip(cached, new, counts):
        o = c % block
        slots += [(first + (o + i) // block, (o + i) % block) for i in range(m)]
        touched += [(first + i // block, i % block) for i in range(o + m if m else 0)]
        first += n
    place = lambda v: ids[_ints([a for a, _ in v], torch.int64)] * block + _ints([b for _, b in v], torch.int64)  # noqa: E731
    tokens = len(slots)
    fused = _randn(g, tokens, 3 * heads, dim)
    fused[..., ::17] *= 4.0
    fused = fused.to(t)
    scale = lambda: (0.01 + 0.02 * torch.rand(blocks, heads, generator=g, device="cuda")) * 2.0  # noqa: E731
    return dict(k=fused[:, heads:2 * heads], v=fused[:, 2 * heads:], slots=place(slots), touched=place(touched),
                k_codes=_codes(g, blocks, heads, block, dim), v_codes=_codes(g, blocks, heads, block, dim), k_scale=scale(), v_scale=scale())


def _attention_inputs(case, seed):
    """A cache whose blocks lie in the order a long-running server leaves them in."""
    g, t = _gen(seed), TYPES[case["dtype"]]
    lens, new = _cache_lengths(case), case["new"]
    heads, dim, block, requests = case["kv_heads"], case["dim"], case["block"], case["requests"]
    need = _ints([-(-v // block) for v in lens])
    blocks, width = int(need.sum()) + 5, int(need.max())
    ids = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(width, device="cuda")
    first = torch.cumsum(need, 0) - need
    table = torch.where(at[None] < need[:, None], ids[(first[:, None] + at[None]).clamp(max=blocks - 1)], 0).to(torch.int32).contiguous()
    q = _randn(g, requests * new, case["group"] * heads, dim).mul_(1.5).to(t)
    scale = lambda: 0.01 + 0.03 * torch.rand(blocks, heads, generator=g, device="cuda")  # noqa: E731
    return dict(q=q, table=table, lens=_ints(lens), starts=_ints([i * new for i in range(requests + 1)]), longest=max(lens),
                k_codes=_codes(g, blocks, heads, block, dim), v_codes=_codes(g, blocks, heads, block, dim), k_scale=scale(), v_scale=scale())


_INPUTS = {"linear": _linear_inputs, "schedule": _schedule_inputs, "append": _append_inputs, "attention": _attention_inputs}
_handle = None


def prepare(case, seed):
    """What a decoding program has in hand: the inputs and, for this package, the plan or the cache that it keeps."""
    global _handle
    state = _INPUTS[case["op"]](case, seed)
    state["case"] = case
    if own:
        from paper_1806_08342_b200 import qtz
        if _handle is None:
            _handle = qtz.Handle(0)
        if case["op"] == "linear":
            state["plan"] = _handle.linear_create(state["codes"], state["scales"], case["k"], case["group"], zeros=state["zeros"], bias=state["bias"])
        elif case["op"] == "schedule":
            state["handle"] = _handle
        else:
            state["cache"] = qtz.KvCache(_handle, state["k_codes"], state["v_codes"], state["k_scale"], state["v_scale"])
    return state


# ---- one pass ----------------------------------------------------------------------------------------------
def run(state):
    return _RUN[state["case"]["op"]](state)


def _linear(s):
    if own:
        return s["plan"](s["x"])
    case = s["case"]
    q = torch.stack((s["codes"] & 15, s["codes"] >> 4), -1).flatten(1)[:, :case["k"]].float()
    group = torch.arange(case["k"], device="cuda") // case["group"]
    q = q - s["zeros"].float()[:, group] if s["zeros"] is not None else torch.where(q > 7, q - 16, q)
    y = torch.matmul(s["x"].float(), (q * s["scales"].float()[:, group]).t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(s["x"].dtype)


def _schedule(s):
    case = s["case"]
    if own:
        starts, lens, slots, report = s["handle"].kv_schedule(s["cached"], s["new"], s["table"], s["free"], s["free_count"], case["block"], s["capacity"])
        return dict(table=s["table"], starts=starts, lens=lens, slots=slots, report=report)
    block, table, free = case["block"], s["table"], s["free"]
    cached, new, count = s["cached"].long(), s["new"].long(), s["free_count"].long()
    lens = cached + new
    have, need = (cached + block - 1) // block, (lens + block - 1) // block
    ends, taken = torch.cumsum(new, 0), torch.cumsum(need - have, 0)
    fits = (taken[-1] <= count[0]) & (need.max() <= table.shape[1]) & (ends[-1] <= s["capacity"])   # all or nothing
    before = taken - (need - have)
    column = torch.arange(table.shape[1], device="cuda")
    from_free = lambda r, j: free[(count - 1 - before[r] - (j - have[r])).clamp(0, free.numel() - 1)]  # noqa: E731
    row = torch.arange(cached.numel(), device="cuda")[:, None]
    fresh = (column >= have[:, None]) & (column < need[:, None]) & fits
    table.copy_(torch.where(fresh, from_free(row, column), table))
    token = torch.arange(s["capacity"], device="cuda")
    r = torch.searchsorted(ends, token, right=True).clamp(max=cached.numel() - 1)
    pos = cached[r] + token - (ends[r] - new[r])
    slots = table[r, (pos // block).clamp(max=table.shape[1] - 1)].long() * block + pos % block
    slots = torch.where((token < ends[-1]) & fits, slots, -1)
    starts = torch.cat((torch.zeros_like(ends[:1]), ends)) * fits
    report = torch.stack((count[0] - taken[-1] * fits, ends[-1] * fits, taken[-1] * fits, 1 - fits.long()))
    return dict(table=table, starts=starts.int(), lens=torch.where(fits, lens, cached).int(), slots=slots, report=report.int())


def _append(s):
    if own:
        s["cache"].append(s["k"], s["v"], s["slots"])
        return s["cache"].read(s["touched"], dtype=s["k"].dtype)
    case, slots, out = s["case"], s["slots"], []
    block, blocks = case["block"], s["k_codes"].shape[0]
    b, o = slots // block, slots % block
    # offset of the block's first new token: what lies before it was there already
    first = torch.full((blocks,), block, device="cuda").scatter_reduce(0, b, o, "amin")
    fresh = first < block
    for x, codes, scale in ((s["k"], s["k_codes"], s["k_scale"]), (s["v"], s["v_codes"], s["v_scale"])):
        x = x.float()
        top = torch.zeros_like(scale).index_reduce(0, b, x.abs().amax(-1), "amax")
        step = (top / torch.full_like(top, 127.0)).clamp(min=MIN_SCALE)
        grown = torch.where((first > 0)[:, None], torch.maximum(step, scale), step)
        ratio = torch.where((fresh & (first > 0))[:, None], scale / grown, torch.ones_like(scale))
        scale.copy_(torch.where(fresh[:, None], grown, scale))
        t = s["touched"]
        tb, to = t // block, t % block
        codes[tb, :, to] = torch.round(codes[tb, :, to].float() * ratio[tb][..., None]).to(torch.int8)
        codes[b, :, o] = torch.clamp(torch.round(x / scale[b][..., None]), -127, 127).to(torch.int8)
        out.append((codes[tb, :, to].float() * scale[tb][..., None]).to(s["k"].dtype))
    return tuple(out)


def _attention(s):
    case = s["case"]
    if own:
        return s["cache"].attention(s["q"], s["starts"], s["lens"], s["table"], window=case["window"], return_lse=True)
    new, heads, group, dim, block = case["new"], case["kv_heads"], case["group"], case["dim"], case["block"]
    requests, length = case["requests"], -(-s["longest"] // block) * block
    table = s["table"].long()
    real = lambda codes, scale: (codes[table].float() * scale[table][..., None, None]).transpose(1, 2).reshape(requests, heads, length, dim)  # noqa: E731
    # rows of one key/value head: (new token, head within the group)
    q = s["q"].float().reshape(requests, new, heads, group, dim).transpose(1, 2).reshape(requests, heads, new * group, dim)
    t = torch.matmul(q, real(s["k_codes"], s["k_scale"]).transpose(-1, -2)) * (1.0 / math.sqrt(dim))
    at = torch.arange(length, device="cuda")
    end = s["lens"].long()[:, None] - new + 1 + torch.arange(new, device="cuda").repeat_interleave(group)
    seen = at < end[..., None]
    if case["window"]:
        seen &= at >= end[..., None] - case["window"]
    t = torch.where(seen[:, None], t, -math.inf)
    top = t.amax(-1, keepdim=True)
    p = torch.exp(t - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    y = torch.matmul(p, real(s["v_codes"], s["v_scale"])) / torch.where(total == 0, 1.0, total)
    back = lambda v: v.reshape(requests, heads, new, group, -1).transpose(1, 2).reshape(requests * new, heads * group, -1)  # noqa: E731
    return back(y).to(s["q"].dtype), back(top + torch.log(total))[..., 0]


_RUN = {"linear": _linear, "schedule": _schedule, "append": _append, "attention": _attention}


# ---- what a pass cannot do without ---------------------------------------------------------------------------
def work(case):
    if case["op"] == "linear":
        rows, n, k = case["rows"], case["n"], case["k"]
        groups = -(-k // case["group"])
        return {"bytes": n * ((k + 1) // 2) + n * groups * (3 if case["zeros"] else 2) + 2 * rows * (n + k) + (2 * n if case["bias"] else 0),
                "flops": 2 * rows * n * k}
    if case["op"] == "attention":
        lens, new, window = _cache_lengths(case), case["new"], case["window"]
        seen = [min(v, window + new - 1) if window else v for v in lens]
        pairs = sum(new * (v if not window else min(v, window)) for v in lens)
        block, heads, dim = case["block"], case["kv_heads"], case["dim"]
        rows = case["requests"] * new * heads * case["group"]
        return {"bytes": sum(2 * heads * (v * dim + -(-v // block) * 4) + -(-v // block) * 4 for v in seen) + rows * (4 * dim + 4),
                "flops": 4 * pairs * heads * case["group"] * dim}
    cached, new = _step_lengths(case)
    block = case["block"]
    if case["op"] == "schedule":
        grown = sum(-(-(c + m) // block) - -(-c // block) for c, m in zip(cached, new))
        return {"bytes": case["requests"] * 16 + 8 * (sum(new) + 7) + 8 * grown, "flops": 0}
    values = sum(new) * case["heads"] * case["dim"]
    touched = sum(c % block + m for c, m in zip(cached, new) if m) * case["heads"] * case["dim"]
    # K and V: new ones read in 16 bits and written in 8; then 8 bits read and 16 written for what was touched
    return {"bytes": 2 * (3 * values + 3 * touched) + 8 * sum(new), "flops": 8 * values}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------
def exact(case, seed):
    return _EXACT[case["op"]](case, _INPUTS[case["op"]](case, seed))


def _exact_linear(case, s):
    n, k, g = case["n"], case["k"], case["group"]
    total = torch.zeros(case["rows"], n, dtype=torch.float64, device="cuda")
    for j in range(-(-k // g)):                               # one group of columns at a time: s * (sum q x - z sum x)
        lo, hi = j * g, min(k, j * g + g)
        x = s["x"][:, lo:hi].double()
        byte = s["codes"][:, lo // 2:(hi + 1) // 2].int()
        q = torch.zeros(n, 2 * byte.shape[1], dtype=torch.float64, device="cuda")
        q[:, 0::2], q[:, 1::2] = byte % 16, byte // 16
        q = q[:, :hi - lo]
        if s["zeros"] is None:
            q = torch.remainder(q + 8, 16) - 8
        part = x @ q.t()
        if s["zeros"] is not None:
            part = part - x.sum(1, keepdim=True) * s["zeros"][:, j].double()
        total += part * s["scales"][:, j].double()
    return total if s["bias"] is None else total + s["bias"].double()


def _exact_append(case, s):
    block, out = case["block"], []
    t = s["touched"]
    for x, codes, scale in ((s["k"], s["k_codes"], s["k_scale"]), (s["v"], s["v_codes"], s["v_scale"])):
        x, scale = x.double(), scale.double()
        b, o = s["slots"] // block, s["slots"] % block
        has_old = torch.ones(codes.shape[0], dtype=torch.bool, device="cuda")
        has_old[b[o == 0]] = False
        step = torch.zeros_like(scale)
        step.index_reduce_(0, b, x.abs().amax(-1) / 127, "amax")
        step.clamp_(min=MIN_SCALE)
        wide = torch.where(has_old[:, None], torch.maximum(step, scale), step)
        q = torch.round(codes.double() * (scale / wide)[:, :, None, None]) * has_old[:, None, None, None]
        q[b, :, o] = torch.round(x / wide[b][..., None]).clamp(-127, 127)
        out.append((q * wide[..., None, None])[t // block, :, t % block])
    return tuple(out)


def _exact_attention(case, s):
    new, heads, group, dim, block = case["new"], case["kv_heads"], case["group"], case["dim"], case["block"]
    y = torch.zeros(case["requests"] * new, heads * group, dim, dtype=torch.float64, device="cuda")
    lse = torch.full(y.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for r, length in enumerate(_cache_lengths(case)):
        ids = s["table"][r, :-(-length // block)].long()
        for h in range(heads):
            k = (s["k_codes"][ids, h].double() * s["k_scale"][ids, h].double()[:, None, None]).flatten(0, 1)
            v = (s["v_codes"][ids, h].double() * s["v_scale"][ids, h].double()[:, None, None]).flatten(0, 1)
            for i in range(new):
                end = length - new + i + 1
                start = max(0, end - case["window"]) if case["window"] else 0
                at, own_heads = r * new + i, slice(h * group, (h + 1) * group)
                t = s["q"][at, own_heads].double() @ k[start:end].t() / math.sqrt(dim)
                lse[at, own_heads] = torch.logsumexp(t, -1)
                y[at, own_heads] = torch.softmax(t, -1) @ v[start:end]
    return y, lse


def _exact_schedule(case, s):
    """By hand, request after request, from the end of the free list."""
    cached, new = _step_lengths(case)
    block, table, free = case["block"], s["table"].tolist(), s["free"].tolist()
    left, slots, starts = len(free), [], [0]
    for r, (c, m) in enumerate(zip(cached, new)):
        for pos in range(c, c + m):
            if table[r][pos // block] < 0:
                left -= 1
                table[r][pos // block] = free[left]
            slots.append(table[r][pos // block] * block + pos % block)
        starts.append(starts[-1] + m)
    report = [left, starts[-1], len(free) - left, 0]
    slots += [-1] * (s["capacity"] - len(slots))
    return dict(table=_ints(table), starts=_ints(starts), lens=_ints([c + m for c, m in zip(cached, new)]), slots=_ints(slots, torch.int64), report=_ints(report))


_EXACT = {"linear": _exact_linear, "schedule": _exact_schedule, "append": _exact_append, "attention": _exact_attention}
