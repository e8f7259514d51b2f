"""4-bit linear layers through the public entry points against fp64.

Bound: products of a code, a scale-free activation and the group's scale are summed in fp32, so the error before the
final rounding is at most 2 (k + 8) 2^-24 sum |x w| (any order of additions, a tensor core's truncation included); the
rounding to the output type adds half a unit in its last place."""
import numpy as np
import pytest
import torch

from gpu_util import hq  # noqa: F401
from oracle import serving
from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu

UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float16, torch.bfloat16)}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}


def make(rows, n, k, group, dtype, zeros, bias, seed, pitch=None):
    g = torch.Generator().manual_seed(seed)
    groups = -(-k // group)
    pitch = -(-k // 8) * 8 if pitch is None else pitch
    x = torch.full((rows, pitch), float("nan"), dtype=dtype)                 # what lies past k must not matter
    x[:, :k] = torch.randn(rows, k, generator=g).to(dtype)
    codes = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, dtype=torch.uint8)
    scales = (torch.rand(n, groups, generator=g) + 0.1).to(dtype)
    z = torch.randint(0, 16, (n, groups), generator=g, dtype=torch.uint8) if zeros else None
    b = torch.randn(n, generator=g).to(dtype) if bias else None
    return x, codes, scales, z, b


def check(y, x, codes, scales, z, b, k, group, signed):
    f = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    x = x[:, :k]
    want = serving.linear(f(x), codes.numpy(), f(scales), None if z is None else z.numpy(), f(b), k, group, signed)
    q = serving.unpack4(codes.numpy(), k, signed).astype(np.float64)
    cols = np.arange(k) // group
    if z is not None:
        q -= z.numpy().astype(np.float64)[:, cols]
    size = np.abs(f(x)) @ np.abs(q * f(scales)[:, cols]).T + (0 if b is None else np.abs(f(b)))
    tol = 2 * (k + 8) * 2.0 ** -24 * size
    tol = tol + UNIT[y.dtype] * (np.abs(want) + tol) + TINY[y.dtype]
    got = f(y.cpu())
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])


CASES = [  # rows, n, k, group
    (1, 16, 64, 32), (1, 1, 1, 32), (1, 17, 31, 32), (1, 1000, 1024, 32), (1, 256, 4096, 128), (2, 40, 65, 64),
    (3, 33, 191, 64), (7, 100, 513, 128), (8, 64, 448, 448), (9, 48, 1000, 64), (13, 321, 777, 32), (16, 128, 256, 256),
    (17, 130, 2050, 128), (31, 65, 640, 64), (32, 512, 1024, 128), (33, 20, 130, 32), (65, 70, 200, 64), (129, 18, 96, 64),
    (1, 4100, 8200, 128), (5, 3, 20011, 192),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_linear_matches_fp64(hq, case, zeros, dtype):
    rows, n, k, group = case
    x, codes, scales, z, b = make(rows, n, k, group, dtype, zeros, (rows + n) % 2 == 0, rows * n + k)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    plan = hq.linear_create(dev(codes), dev(scales), k, group, zeros=dev(z), bias=dev(b))
    y = plan(dev(x)[:, :k])
    check(y, x, codes, scales, z, b, k, group, not zeros)
    assert torch.equal(plan(dev(x)[:, :k]), y)                               # the same bits when repeated
    plan.close()


def test_unsigned_codes_without_zero_points_and_large_zero_points(hq):
    x, codes, scales, z, _ = make(4, 50, 200, 64, torch.bfloat16, True, False, 3)
    y = hq.linear_create(codes.cuda(), scales.cuda(), 200, 64, signed=False)(x.cuda()[:, :200])
    check(y, x, codes, scales, None, None, 200, 64, False)
    big = z + 13                                                              # 16 .. 28 count as 15
    y = hq.linear_create(codes.cuda(), scales.cuda(), 200, 64, zeros=big.cuda())(x.cuda()[:, :200])
    check(y, x, codes, scales, torch.minimum(big, torch.tensor(15, dtype=torch.uint8)), None, 200, 64, False)


def test_values_at_the_ends_of_the_types(hq):
    """Activations and scales near the types' ends: nothing in between may overflow or be flushed."""
    for dtype, top in ((torch.float16, 60000.0), (torch.bfloat16, 1e34)):
        x, codes, scales, _, _ = make(2, 32, 128, 64, dtype, False, False, 11)
        x[0] = x[0] * 0 + top
        x[1, :128] = torch.tensor([2.0 ** -14, -(2.0 ** -20)]).repeat(64).to(dtype)
        scales = torch.full_like(scales, 2.0 ** -14)
        y = hq.linear_create(codes.cuda(), scales.cuda(), 128, 64)(x.cuda())
        check(y[1:], x[1:], codes, scales, None, None, 128, 64, True)
        x[0, :128] = top
        y = hq.linear_create(codes.cuda(), scales.cuda(), 128, 64)(x.cuda())
        check(y, x, codes, scales, None, None, 128, 64, True)


def test_nan_and_infinity_stay_in_their_row(hq):
    x, codes, scales, _, _ = make(3, 40, 256, 128, torch.float16, False, False, 12)
    x[1, 7] = float("nan")
    y = hq.linear_create(codes.cuda(), scales.cuda(), 256, 128)(x.cuda()).cpu()
    assert torch.isnan(y[1]).all()                                             # NaN * 0 is NaN too
    check(y[::2], x[::2], codes, scales, None, None, 256, 128, True)


def test_strides_leading_axes_out_and_streams(hq):
    rows, n, k = 6, 77, 320
    x, codes, scales, _, b = make(rows, n, k, 64, torch.bfloat16, False, True, 21, pitch=352)
    plan = hq.linear_create(codes.cuda(), scales.cuda(), k, 64, bias=b.cuda())
    wide = torch.full((rows, 100), 7.0, dtype=torch.bfloat16, device="cuda")
    xd = x.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan(xd[:, :k], out=wide[:, 5:5 + n])
    torch.cuda.current_stream().wait_stream(side)
    check(wide[:, 5:5 + n], x, codes, scales, None, b, k, 64, True)
    assert (wide[:, :5] == 7).all() and (wide[:, 5 + n:] == 7).all()
    y = plan(xd[:, :k].contiguous().view(2, 3, k))
    assert y.shape == (2, 3, n) and torch.equal(y.view(rows, n), wide[:, 5:5 + n])
    assert plan(xd[:0, :k]).shape == (0, n)
    graph = torch.cuda.CUDAGraph()
    out = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    with torch.cuda.graph(graph):
        plan(xd[:, :k], out=out)
    graph.replay()
    assert torch.equal(out, y.view(rows, n))


def test_group_quantizer_feeds_the_layer(hq):
    g = torch.Generator().manual_seed(31)
    for symmetric, k, group, dtype in ((True, 256, 64, torch.bfloat16), (False, 256, 32, torch.float16), (True, 203, 64, torch.float16),
                                       (False, 130, 128, torch.bfloat16)):
        w = torch.randn(24, k, generator=g) * torch.rand(24, 1, generator=g)
        codes, scales, zeros = hq.quantize_groups(w.cuda(), group, dtype, symmetric)
        assert codes.shape == (24, (k + 1) // 2) and (zeros is None) == symmetric
        q = serving.unpack4(codes.cpu().numpy(), k, symmetric).astype(np.float64)
        cols = np.arange(k) // group
        if zeros is not None:
            q -= zeros.cpu().numpy().astype(np.float64)[:, cols]
        s = scales.cpu().double().numpy()[:, cols]
        # half a step; the rounded scale may leave the largest value of a group up to 7.5 * 2^-8 steps (15.5 * 2^-8 unsigned) outside
        assert (np.abs(q * s - w.double().numpy()) <= s * (0.5 + 16 * 2.0 ** -8)).all()
        x = torch.randn(3, (k + 7) // 8 * 8, generator=g).to(dtype)
        y = hq.linear_create(codes, scales, k, group, zeros=zeros)(x.cuda()[:, :k])
        check(y, x, codes.cpu(), scales.cpu(), None if zeros is None else zeros.cpu(), None, k, group, symmetric)


def test_refusals(hq):
    x, codes, scales, z, b = (None if t is None else t.cuda() for t in make(2, 32, 128, 64, torch.float16, True, True, 41))
    for bad_group, code in ((48, -3), (16, -3), (0, None), (-64, None)):
        with pytest.raises((qtz.QtzError, ValueError)) as e:
            hq.linear_create(codes, torch.ones(32, -(-128 // bad_group) if bad_group > 0 else 2, dtype=torch.float16, device="cuda"), 128, bad_group)
        if code:
            assert e.value.code == code
    with pytest.raises(ValueError):
        hq.linear_create(codes, scales.float(), 128, 64)
    with pytest.raises(ValueError):
        hq.linear_create(codes[:, :-1].contiguous(), scales, 128, 64)
    with pytest.raises(ValueError):
        hq.linear_create(codes.cpu(), scales, 128, 64)
    with pytest.raises(qtz.QtzError) as e:
        hq.linear_create(codes, scales, 128, 64, zeros=z, signed=True)
    assert e.value.code == -1
    plan = hq.linear_create(codes, scales, 128, 64, zeros=z, bias=b)
    with pytest.raises(ValueError):
        plan(x.bfloat16())
    with pytest.raises(ValueError):
        plan(x[:, :64])
    with pytest.raises(qtz.QtzError) as e:                                     # a base and a stride off 16 bytes
        plan(torch.zeros(2 * 128 + 1, dtype=torch.float16, device="cuda")[1:].view(2, 128))
    assert e.value.code == -2
    with pytest.raises(qtz.QtzError) as e:
        plan(torch.zeros(2, 130, dtype=torch.float16, device="cuda")[:, :128])
    assert e.value.code == -2
    lib = qtz.load_library()
    assert lib.qtz_linear_w4(None, x.data_ptr(), 128, 2, x.data_ptr(), 32, None) == -1
    assert lib.qtz_linear_w4(plan.plan, x.data_ptr(), 120, 2, x.data_ptr(), 32, None) == -1
    assert lib.qtz_linear_w4(plan.plan, x.data_ptr(), 128, -1, x.data_ptr(), 32, None) == -1
    assert lib.qtz_linear_w4(plan.plan, None, 128, 2, x.data_ptr(), 32, None) == -1
    assert lib.qtz_linear_w4(plan.plan, x.data_ptr(), 128, 2, x.data_ptr(), 31, None) == -1
    assert lib.qtz_linear_destroy(None) == -1
