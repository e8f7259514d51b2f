"""4-bit linear layers where activations are not finite."""
import numpy as np
import pytest
import torch

from gpu_util import hq  # noqa: F401

pytestmark = pytest.mark.gpu


def layer(hq, g, n, k, group, dtype, zeros):
    groups = -(-k // group)
    codes = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, dtype=torch.uint8)
    scales = (torch.rand(n, groups, generator=g) + 0.1).to(dtype)
    z = torch.randint(0, 16, (n, groups), generator=g, dtype=torch.uint8) if zeros else None
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(1)[:, :k].double()
    at = torch.arange(k) // group
    q = q - z[:, at].double() if zeros else torch.where(q > 7, q - 16, q)
    plan = hq.linear_create(codes.cuda(), scales.cuda(), k, group, zeros=None if z is None else z.cuda())
    return plan, q * scales.double()[:, at]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 7, 8, 9, 17, 33])
@pytest.mark.parametrize("n,k,group,zeros", [(40, 256, 128, False), (300, 777, 32, True), (257, 2049, 64, False), (33, 600, 192, True)])
def test_infinities_and_nan_as_in_the_definition(hq, n, k, group, zeros, rows, dtype):
    """Each output is what sums of products of reals with infinities give, whatever the number of rows: an infinity, NaN where two of
    them differ in sign or meet a weight of zero, and finite values in the rows beside."""
    g = torch.Generator().manual_seed(n + rows)
    plan, w = layer(hq, g, n, k, group, dtype, zeros)
    x = torch.randn(rows, -(-k // 8) * 8, generator=g).to(dtype)[:, :k]
    x[0, 7 % k] = float("inf")
    if rows > 2:
        x[1, k - 1] = -float("inf")
    if rows > 3:
        x[2, [3, 5, k // 2]] = torch.tensor([float("inf"), -float("inf"), float("inf")], dtype=dtype)
    if rows > 4:
        x[3, k // 3] = float("nan")
        x[4, [1, 4, k - 2]] = float("inf")
    want = np.empty((rows, n))
    with np.errstate(invalid="ignore"):
        for r in range(rows):                                       # no product that the definition does not have
            want[r] = (x[r].double().numpy() * w.numpy()).sum(1)
    padded = torch.zeros(rows, -(-k // 8) * 8, dtype=dtype)
    padded[:, :k] = x
    got = plan(padded.cuda()[:, :k]).double().cpu().numpy()
    odd = ~np.isfinite(want)
    assert odd[0].all() and np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    size = np.abs(np.nan_to_num(x.double().numpy(), nan=0, posinf=0, neginf=0)) @ np.abs(w.numpy()).T
    tol = 2 * (k + 8) * 2.0 ** -24 * size
    tol = tol + torch.finfo(dtype).eps / 2 * (np.abs(np.where(odd, 0, want)) + tol) + 2.0 ** -25
    assert (np.abs(got[~odd] - want[~odd]) <= tol[~odd]).all()


@pytest.mark.parametrize("dtype,strong", [(torch.float16, 2.0 ** 15), (torch.bfloat16, 2.0 ** 20)])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 12])
@pytest.mark.parametrize("n,k,group,zeros", [(300, 512, 64, False), (70, 777, 32, True), (64, 256, 128, False)])
def test_strong_values_that_meet_weights_of_zero(hq, n, k, group, zeros, rows, dtype, strong):
    """One value of each row lies far above the others, and half of the weights that it meets are zero: there the others are all that
    counts.  Bound: that of fp32 sums, 2 (k + 8) 2^-24 sum |x w|, half of 2^-29 of the strong value for each column of a block of 256
    (no sum is off by more), and the rounding to the output's type."""
    g = torch.Generator().manual_seed(n + rows)
    at = 5
    codes = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, dtype=torch.uint8)
    scales = (torch.rand(n, -(-k // group), generator=g) + 0.1).to(dtype)
    z = torch.randint(1, 15, (n, -(-k // group)), generator=g, dtype=torch.uint8) if zeros else None
    none = z[::2, at // group] if zeros else torch.zeros((n + 1) // 2, dtype=torch.uint8)
    codes[::2, at // 2] = (codes[::2, at // 2] & 15) | (none << 4)             # column 5 is a high nibble
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(1)[:, :k].double()
    cols = torch.arange(k) // group
    w = (q - z[:, cols].double() if zeros else torch.where(q > 7, q - 16, q)) * scales.double()[:, cols]
    assert not w[::2, at].any()
    x = torch.randn(rows, -(-k // 8) * 8, generator=g).to(dtype)
    x[:, at] = strong
    got = hq.linear_create(codes.cuda(), scales.cuda(), k, group, zeros=None if z is None else z.cuda())(x.cuda()[:, :k]).double().cpu()
    x = x[:, :k].double()
    want = x @ w.T
    tol = 2 * (k + 8) * 2.0 ** -24 * (x.abs() @ w.abs().T) + 2.0 ** -30 * strong * w[:, :256].abs().sum(1)
    tol = tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol) + 2.0 ** -25
    worst = ((got - want).abs() / tol)[torch.isfinite(got)].max().item()
    assert worst <= 1.0 and bool(torch.isfinite(got[:, ::2]).all()), worst
