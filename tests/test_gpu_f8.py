"""Norm and quantizers of the 8-bit floating-point operators through the public entry points against fp64.

Bounds.  A value of the norm is off by at most 2^-18 of itself before it is rounded: a sum of at most 32768 squares in fp32 takes at most
32 steps a thread and ten to join them, whose roundings the square root halves, and a handful of roundings follow.  A gated value is off
by at most 2^-16: the exponential by 105 units at a gate of -88, the division by two, three products.  Scales add one rounding.  A code is
within half a step of the value over the scale, and within what value and scale are off by."""
import numpy as np
import pytest
import torch

from gpu_util import hq  # noqa: F401
from oracle import f8
from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu

UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.float16, torch.bfloat16)}
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = list(UNIT)


def f64(t):
    return t.double().cpu().numpy()


def inside(rows, k, dtype, fill=float("nan"), multiple=8, more=8):
    """A view [rows][k] into a wider tensor whose other places hold `fill`."""
    wide = torch.full((rows, (k + multiple - 1) // multiple * multiple + more), fill, dtype=dtype, device="cuda")
    return wide, wide[:, :k]


def check_codes(codes, scales, v, off, rows=1):
    """Codes and scales of values v that are known within a part `off` of themselves."""
    n, k = v.shape
    s, want = f64(scales), f8.scales(v, rows)
    assert s.shape == want.shape
    assert (np.abs(s - want) <= want * (off + 2.0 ** -23)).all(), np.abs(s / want - 1).max()
    got = f8.decode(codes.contiguous().view(torch.uint8).cpu().numpy())
    finite = np.isfinite(v)
    assert np.array_equal(np.isnan(got), np.isnan(v))
    q = np.where(finite, v, 0.0) / f8.spread(s, n, k, rows)
    bad = finite & ~(np.abs(got - q) <= f8.half_step(np.minimum(np.abs(q), 447.0)) + np.abs(q) * (off + 2.0 ** -22))
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], q[bad][:4])
    assert (got[np.isinf(v)] == np.sign(v[np.isinf(v)]) * 448).all()


def check_norm(outputs, x, gain, eps, residual):
    codes, scales, values, total = outputs
    want_sum, want = f8.rmsnorm(f64(x), f64(gain), eps, None if residual is None else f64(residual))
    if codes is not None:
        check_codes(codes, scales, want, 2.0 ** -18)
    for got, w, off in ((values, want, 2.0 ** -18), (total, want_sum, 2.0 ** -24)):
        if got is not None:
            assert got.dtype is x.dtype
            tol = np.abs(w) * (off + UNIT[x.dtype] * 1.001) + TINY[x.dtype]
            assert (np.abs(f64(got) - w) <= tol).all()


WIDTHS = [1, 7, 8, 31, 64, 127, 128, 129, 250, 1000, 1024, 2048, 5003, 8192, 8193, 10001, 16385, 32768]


@pytest.mark.parametrize("k", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 3, 400])
def test_norm_matches_fp64(hq, rows, k, dtype):
    if rows == 400 and k > 10001:
        rows = 299                                                       # still more than one row a CTA's place
    g = torch.Generator("cuda").manual_seed(rows * k)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    _, x = inside(rows, k, dtype)
    _, residual = inside(rows, k, dtype, more=16)
    x.copy_(rand(rows, k))
    residual.copy_(rand(rows, k) * 4)
    gain = (1 + 0.3 * rand(k)).to(dtype)
    for res in (None, residual):
        out = hq.f8_rmsnorm(x, gain, 1e-5, residual=res, values=True)
        check_norm(out, x, gain, 1e-5, res)
        again = hq.f8_rmsnorm(x, gain, 1e-5, residual=res)
        assert torch.equal(again[0].view(torch.uint8), out[0].view(torch.uint8)) and torch.equal(again[1], out[1]) and again[2] is None
        assert (again[3] is None) == (res is None)
        only = hq.f8_rmsnorm(x, gain, 1e-5, residual=res, codes=False, values=True)
        assert only[0] is None and only[1] is None and torch.equal(only[2], out[2])


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_odd_rows(hq, dtype):
    """Zeros, tiny and huge values, infinities, NaN, a block of zeros in a row that has others; every row for itself."""
    k, big = 300, float(torch.finfo(dtype).max)
    x = torch.randn(9, k, device="cuda").to(dtype)
    x[1] = 0
    x[2] *= 1e-4
    x[3] = big
    x[4, 7] = big
    x[5, 9] = float("inf")
    x[6, 11] = float("nan")
    x[7, 128:256] = 0
    x[8] = big / 1e3
    wide, view = inside(9, k, dtype)
    view.copy_(x)
    gain = torch.ones(k, device="cuda", dtype=dtype)
    codes, scales, values, _ = hq.f8_rmsnorm(view, gain, 1e-6, values=True)
    want_sum, want = f8.rmsnorm(f64(x), f64(gain), 1e-6)
    usual = [0, 1, 2, 3, 4, 7, 8]
    check_codes(codes[usual], scales[usual], want[usual], 2.0 ** -18)
    assert (np.abs(f64(values)[usual] - want[usual]) <= np.abs(want[usual]) * (2.0 ** -18 + UNIT[dtype] * 1.001) + TINY[dtype]).all()
    row = f64(values)[5]
    assert np.isnan(row[9]) and (np.delete(row, 9) == 0).all() and np.isnan(f64(values)[6]).all()
    assert np.isnan(f8.decode(codes.contiguous().view(torch.uint8).cpu().numpy()[6])).all() and (f64(scales)[6] == 2.0 ** -100).all()
    assert (f64(scales)[1] == 2.0 ** -100).all() and (f64(scales)[7, 1] == 2.0 ** -100)


def test_norm_writes_into_its_residual_and_nothing_past_a_row(hq):
    g = torch.Generator("cuda").manual_seed(5)
    x = torch.randn(5, 204, device="cuda", generator=g).bfloat16()
    for k in (200, 201, 203):
        wide, residual = inside(5, k, torch.bfloat16, fill=7.0)
        pitch = wide.shape[1]
        residual.copy_(torch.randn(5, k, device="cuda", generator=g))
        xs = torch.zeros(5, 208, device="cuda", dtype=torch.bfloat16)[:, :k].copy_(x[:, :k])
        gain = torch.rand(k, device="cuda", generator=g).bfloat16()
        before = residual.clone()
        apart = hq.f8_rmsnorm(xs, gain, residual=residual, values=True)
        assert torch.equal(residual, before)
        got = hq.f8_rmsnorm(xs, gain, residual=residual, values=True, sum_out=residual)
        assert got[3] is residual and torch.equal(residual, apart[3]) and torch.equal(got[0].view(torch.uint8), apart[0].view(torch.uint8))
        assert bool((wide[:, k:] == 7).all()) and wide.shape[1] == pitch


@pytest.mark.parametrize("k", WIDTHS[:-1])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 5, 700])
def test_quantize_matches_fp64(hq, rows, k, dtype):
    g = torch.Generator("cuda").manual_seed(rows + 3 * k)
    _, x = inside(rows, k, dtype)
    _, gate = inside(rows, k, dtype, more=24)
    x.copy_(torch.randn(rows, k, device="cuda", generator=g) * 10)
    gate.copy_(torch.randn(rows, k, device="cuda", generator=g) * 3)
    check_codes(*hq.f8_quantize(x), f64(x), 0.0)
    check_codes(*hq.f8_quantize(x, gate=gate), f8.gated(f64(x), f64(gate)), 2.0 ** -16)


def test_quantize_far_gates_and_special_values(hq):
    gate = torch.tensor([0.0, -0.0, 1e-6, -1e-6, 20.0, -20.0, 60.0, -60.0, 88.0, -88.0, 1000.0, -1000.0, float("inf"), 3e38, -3e38, 5.0],
                        device="cuda").repeat(8)
    x = torch.linspace(0.5, 2.0, 128, device="cuda")
    rows = torch.stack([x, x * 1e30, x * 1e-30])
    for j in range(16):                                                  # each gate in a block of its own, so that its scale is its own
        one = gate[j].expand(3, 128).contiguous()
        if j in (12, 13):
            continue
        check_codes(*hq.f8_quantize(rows, gate=one), np.where(np.abs(f64(one)) > 88.7, np.where(f64(one) > 0, f8.gated(f64(rows), f64(one)), 0.0),
                                                              f8.gated(f64(rows), f64(one))), 2.0 ** -16)
    v = torch.randn(4, 256, device="cuda")
    v[0, 3], v[1, 200], v[2, 5], v[3, :128] = float("inf"), -float("inf"), float("nan"), 0.0
    check_codes(*hq.f8_quantize(v), f64(v), 0.0)
    v = torch.full((1, 128), float("nan"), device="cuda")
    codes, scales = hq.f8_quantize(v)
    assert bool(codes.float().isnan().all()) and float(scales) == 2.0 ** -100
    tiny = torch.full((1, 128), 2.0 ** -130, device="cuda")
    codes, scales = hq.f8_quantize(tiny)
    assert float(scales) == 2.0 ** -100 and bool((codes.float() == 0).all())


def test_ties_go_to_the_even_code(hq):
    """With a largest value of 448 the scale is 1: what lies half way between two codes is known exactly."""
    values = f8.decode(np.arange(127))
    middle = (values[1:] + values[:-1]) / 2
    v = torch.zeros(1, 128, device="cuda")
    v[0, :126] = torch.from_numpy(middle).float()
    v[0, 127] = 448.0
    codes, scales = hq.f8_quantize(v)
    assert float(scales) == 1.0
    got = codes.view(torch.uint8)[0, :126].cpu().numpy().astype(int)
    low = np.arange(126)
    assert np.array_equal(got, low + low % 2)


@pytest.mark.parametrize("shape", [(1, 1), (1, 500), (129, 127), (128, 128), (300, 1000), (5, 130)])
@pytest.mark.parametrize("dtype", TYPES)
def test_weights_match_fp64(hq, shape, dtype):
    g = torch.Generator("cuda").manual_seed(shape[0])
    w = torch.randn(shape[0], shape[1] + 3, device="cuda", generator=g).to(dtype)[:, 1:-2]
    codes, scales = hq.f8_quantize_weights(w)
    check_codes(codes, scales, f64(w), 0.0, 128)


def test_no_rows(hq):
    x = torch.empty(0, 256, device="cuda")
    codes, scales, values, _ = hq.f8_rmsnorm(x, torch.ones(256, device="cuda"), values=True)
    assert codes.shape == (0, 256) and scales.shape == (0, 2) and values.shape == (0, 256)
    assert hq.f8_quantize(x, gate=x)[0].shape == (0, 256)


def test_rows_beyond_32_bits(hq):
    """Offsets of rows past 2^31 elements: the last rows of a tall tensor."""
    rows, k = 70001, 32768
    x = torch.zeros(rows, k, device="cuda", dtype=torch.bfloat16)
    x[-2:] = torch.randn(2, k, device="cuda").bfloat16()
    codes, scales = hq.f8_quantize(x)
    check_codes(codes[-2:], scales[-2:], f64(x[-2:]), 0.0)
    assert bool((scales[:-2] == 2.0 ** -100).all())
    del codes, scales
    gain = torch.ones(k, device="cuda", dtype=torch.bfloat16)
    codes, scales, _, total = hq.f8_rmsnorm(x, gain, residual=x, sum_out=x)
    check_codes(codes[-2:], scales[-2:], f8.rmsnorm(f64(total[-2:]) / 2, f64(gain), 0.25e-6, None)[1], 2.0 ** -18)
    torch.cuda.empty_cache()


def test_refusals(hq):
    x, gain = torch.zeros(4, 256, device="cuda"), torch.ones(256, device="cuda")
    for call in (lambda: hq.f8_rmsnorm(x.double(), gain), lambda: hq.f8_rmsnorm(x[0], gain), lambda: hq.f8_rmsnorm(x, gain[:-1]),
                 lambda: hq.f8_rmsnorm(x, gain.half()), lambda: hq.f8_rmsnorm(x, gain, residual=x[:3]), lambda: hq.f8_rmsnorm(x, gain, sum_out=x),
                 lambda: hq.f8_rmsnorm(x.t(), torch.ones(4, device="cuda")), lambda: hq.f8_rmsnorm(x, gain.cpu()), lambda: hq.f8_rmsnorm(x.cpu(), gain),
                 lambda: hq.f8_quantize(x, gate=x.half()), lambda: hq.f8_quantize(x.int()), lambda: hq.f8_quantize(x, gate=x[:, :255]),
                 lambda: hq.f8_quantize_weights(x[0]), lambda: hq.f8_quantize_weights(x.int())):
        with pytest.raises(ValueError):
            call()
    flat = torch.zeros(4096, device="cuda")
    shifted, odd = flat[1:1025].view(4, 256), flat[:4 * 257].view(4, 257)[:, :256]
    for call, code in ((lambda: hq.f8_rmsnorm(shifted, gain), -2), (lambda: hq.f8_rmsnorm(odd, gain), -2), (lambda: hq.f8_rmsnorm(x, flat[1:257]), -2),
                       (lambda: hq.f8_quantize(shifted), -2), (lambda: hq.f8_quantize(x, gate=odd), -2), (lambda: hq.f8_rmsnorm(x, gain, eps=0.0), -1),
                       (lambda: hq.f8_rmsnorm(x, gain, eps=float("nan")), -1), (lambda: hq.f8_rmsnorm(x, gain, codes=False), -1),
                       (lambda: hq.f8_rmsnorm(torch.zeros(1, 32776, device="cuda"), torch.zeros(32776, device="cuda")), -9)):
        with pytest.raises(qtz.QtzError) as e:
            call()
        assert e.value.code == code
    assert hq.f8_quantize(odd[:1])[0].shape == (1, 256)                  # a single row has no stride to keep
