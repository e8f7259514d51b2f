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
