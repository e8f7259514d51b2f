"""Linear layers in 8-bit floating point through the public entry points against fp64.

Bound: products of codes are exact; they and the scaled sums of the blocks are summed in fp32, so the error before the final rounding is at
most 2 (k + 8) 2^-24 sum |x w| (any order of additions, a tensor core's truncation included); the rounding to the output type adds half a
unit in its last place."""
import numpy as np
import pytest
import torch

from gpu_util import hq  # noqa: F401
from oracle import f8
from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu

UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.float16, torch.bfloat16)}
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def random_codes(g, *shape):
    """Codes of every exponent and sign, no NaN."""
    c = torch.randint(0, 256, shape, device="cuda", generator=g, dtype=torch.uint8)
    return torch.where((c & 127) == 127, c - 1, c)


def make(rows, n, k, seed, pitch=None):
    g = torch.Generator("cuda").manual_seed(seed)
    pitch = -(-k // 16) * 16 if pitch is None else pitch
    x = torch.full((rows, pitch), 0x7f, device="cuda", dtype=torch.uint8)      # NaN past k must not matter
    x[:, :k] = random_codes(g, rows, k)
    w = random_codes(g, n, k)
    rand = lambda *s: torch.rand(*s, device="cuda", generator=g) + 0.25  # noqa: E731
    return x.view(qtz.E4M3)[:, :k], rand(rows, -(-k // 128)), w.view(qtz.E4M3), rand(-(-n // 128), -(-k // 128)) * 2.0 ** -12, torch.randn(n, device="cuda", generator=g)


def host(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def check(y, x, xs, w, ws, bias, rows=None):
    pick = slice(None) if rows is None else rows
    want, size = f8.linear(host(x[pick]), xs[pick].cpu().numpy(), host(w), ws.cpu().numpy(), None if bias is None else bias.double().cpu().numpy())
    tol = 2 * (w.shape[1] + 8) * 2.0 ** -24 * size
    tol = tol + UNIT[y.dtype] * (np.abs(want) + tol) + TINY[y.dtype]
    got = y[pick].double().cpu().numpy()
    over = np.abs(want) > torch.finfo(y.dtype).max * (1 - UNIT[y.dtype])         # fp16: beyond the type
    assert got.shape == want.shape and np.isinf(got[over]).all()
    bad = ~(np.abs(got - want) <= tol) & ~over
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])


CASES = [  # rows, n, k
    (1, 1, 1), (1, 17, 31), (1, 1000, 1024), (1, 128, 128), (2, 129, 127), (3, 40, 65), (5, 300, 2000), (8, 4100, 512), (15, 256, 640), (16, 256, 4096),
    (17, 130, 2050), (31, 65, 640), (32, 512, 1024), (33, 20, 130), (48, 1000, 3001), (63, 257, 384), (64, 2048, 2048), (65, 70, 200), (96, 640, 1500),
    (127, 128, 256), (128, 384, 129), (129, 18, 96), (200, 1000, 1111), (255, 513, 512), (256, 256, 1024), (257, 768, 333), (300, 5003, 700),
    (511, 300, 1300), (512, 1024, 1024), (1000, 1001, 999), (1777, 640, 384), (2049, 257, 130), (1, 3, 20011), (40, 129, 16000),
]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("dtype", list(UNIT))
def test_linear_matches_fp64(hq, case, dtype):
    rows, n, k = case
    x, xs, w, ws, bias = make(rows, n, k, rows * n + k)
    bias = bias.to(dtype) if rows % 2 else None
    plan = hq.f8_linear_create(w, ws, bias=bias)
    y = plan(x, xs, dtype=dtype)
    check(y, x, xs, w, ws, bias)
    assert torch.equal(plan(x, xs, dtype=dtype), y)                            # the same bits when repeated
    assert hq.device_status() == (0, 0)
    plan.close()


@pytest.mark.parametrize("rows", [1, 20, 100, 700])
def test_strides_of_codes_scales_and_outputs(hq, rows):
    n, k = 333, 700
    x, xs, w, ws, bias = make(rows, n, k, 4, pitch=768)
    apart = torch.zeros(n, k + 5, device="cuda", dtype=torch.uint8)
    apart[:, 3:3 + k] = w.view(torch.uint8)
    plan = hq.f8_linear_create(apart.view(qtz.E4M3)[:, 3:3 + k], ws, bias=bias)   # rows of weights need not touch, nor start on 16 bytes
    want = plan(x, xs, dtype=torch.float32)
    check(want, x, xs, w, ws, bias)
    turned = xs.t().contiguous().t()
    spread = torch.full((rows, 3 * xs.shape[1] + 1), float("nan"), device="cuda")[:, 1::3]
    spread.copy_(xs)
    for scales in (turned, spread):
        assert torch.equal(plan(x, scales, dtype=torch.float32), want)
    wide = torch.full((rows + 2, n + 9), 7.0, device="cuda", dtype=torch.bfloat16)
    for shift in (0, 1, 8):                                                     # any alignment of y
        wide.fill_(7)
        out = wide[1:-1, shift:shift + n]
        assert plan(x, xs, out=out) is out
        assert torch.equal(out, want.bfloat16())
        out.fill_(7)
        assert bool((wide == 7).all())                                          # nothing beside it was written
    same = xs[:1].expand(rows, -1)                                              # one row of scales for all
    check(plan(x, same, dtype=torch.float32), x, same, w, ws, bias)


@pytest.mark.parametrize("rows", [1, 40, 150, 600])
def test_large_and_small_products_in_one_sum(hq, rows):
    """Sums whose largest products cancel, in one block and across blocks."""
    n, k = 200, 512
    x = torch.full((rows, k), 2.0 ** -9, device="cuda").to(qtz.E4M3)
    w = torch.full((n, k), 2.0 ** -3, device="cuda").to(qtz.E4M3)
    x[:, 5], x[:, 300] = 448.0, 448.0
    w[:, 5], w[:, 300] = 448.0, -448.0
    xs, ws = torch.ones(rows, 4, device="cuda"), torch.ones(2, 4, device="cuda")
    check(hq.f8_linear_create(w, ws)(x, xs, dtype=torch.float32), x, xs, w, ws, None)
    x[:, 300], x[:, 6], w[:, 6] = 2.0 ** -9, 448.0, -448.0                      # in one block
    w[:, 300] = 2.0 ** -3
    check(hq.f8_linear_create(w, ws)(x, xs, dtype=torch.float32), x, xs, w, ws, None)


@pytest.mark.parametrize("rows", [1, 40, 150, 600])
def test_nan_codes_stay_in_their_row_and_column(hq, rows):
    n, k = 260, 300
    x, xs, w, ws, _ = make(rows, n, k, 9)
    clean = hq.f8_linear_create(w, ws)(x, xs, dtype=torch.float32)
    x.view(torch.uint8)[rows // 2, 131] = 0x7f                                  # in place: a clone's rows would not start on 16 bytes
    w.view(torch.uint8)[77, 299] = 0xff
    y = hq.f8_linear_create(w, ws)(x, xs, dtype=torch.float32)
    lost = torch.zeros_like(y, dtype=torch.bool)
    lost[rows // 2], lost[:, 77] = True, True
    assert torch.equal(y.isnan(), lost) and torch.equal(y[~lost], clean[~lost])


def test_scales_of_empty_blocks_and_far_scales(hq):
    """Blocks of zeros have the least scale, 2^-100: products of two of them pass below fp32 and count as nothing."""
    x, xs, w, ws, _ = make(30, 300, 512, 2)
    x, w = x.clone(), w.clone()
    x[:, 128:256], xs[:, 1] = 0.0, 2.0 ** -100
    w[128:256, 128:256], ws[1, 1] = 0.0, 2.0 ** -100
    xs[:, 2], ws[:, 2] = 2.0 ** 60, 2.0 ** -70
    check(hq.f8_linear_create(w, ws)(x, xs, dtype=torch.float32), x, xs, w, ws, None)


def test_no_rows_and_refusals(hq):
    x, xs, w, ws, bias = make(4, 256, 256, 1)
    plan = hq.f8_linear_create(w, ws, bias=bias)
    assert plan(x[:0], xs[:0]).shape == (0, 256)
    for call in (lambda: plan(x[:, :255], xs), lambda: plan(x, xs[:, :1]), lambda: plan(x.view(torch.uint8), xs), lambda: plan(x, xs.double()),
                 lambda: plan(x, xs, dtype=torch.float64), lambda: plan(x, xs, out=torch.empty(4, 255, device="cuda")), lambda: plan(x.cpu(), xs),
                 lambda: plan(x, xs, out=torch.empty(256, 4, device="cuda").t()), lambda: plan(x[:, ::2], xs), lambda: plan(x, xs[:3]),
                 lambda: hq.f8_linear_create(w[0], ws), lambda: hq.f8_linear_create(w, ws[:1]), lambda: hq.f8_linear_create(w, ws.half()),
                 lambda: hq.f8_linear_create(w.view(torch.uint8), ws), lambda: hq.f8_linear_create(w, ws, bias=bias[:-1]),
                 lambda: hq.f8_linear_create(w, ws, bias=bias.double()), lambda: hq.f8_linear_create(w.t(), ws)):
        with pytest.raises(ValueError):
            call()
    flat = torch.zeros(4096, device="cuda", dtype=torch.uint8).view(qtz.E4M3)
    for bad in (flat[1:1025].view(4, 256), flat[:4 * 257].view(4, 257)[:, :256]):
        with pytest.raises(qtz.QtzError) as e:
            plan(bad, xs)
        assert e.value.code == -2
    plan.close()


def test_plan_outlives_its_inputs_and_its_handle():
    h = qtz.Handle(0)
    x, xs, w, ws, bias = make(20, 300, 300, 3)
    keep = [t.clone() for t in (w, ws, bias)]
    plan = h.f8_linear_create(w, ws, bias=bias)
    for t in (w.view(torch.uint8), ws, bias):
        t.zero_()
    check(plan(x, xs), x, xs, *keep)
    h.close()
    with pytest.raises(ValueError):
        plan(x, xs)
    plan.close()
