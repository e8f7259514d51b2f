"""Norms of rows whose squares pass fp32: small values beside large ones keep their bits."""
import pytest
import torch

from gpu_util import hq  # noqa: F401
from test_gpu_f8 import check_norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [3, 300, 5003, 20000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("largest", [1e20, 1e27, 3e38])
def test_small_values_beside_large_ones(hq, dtype, largest, k):
    """Values from 2^-115 of the largest to the largest itself: v is above the least normal fp32 number, whatever the row is scaled by on the way."""
    g = torch.Generator("cuda").manual_seed(k)
    x = largest * torch.exp2(-115 * torch.rand(5, k, device="cuda", generator=g)) * torch.sign(torch.randn(5, k, device="cuda", generator=g))
    x[:, 0], x[1, 2] = largest, -largest
    wide = torch.zeros(5, (k + 7) // 8 * 8, device="cuda", dtype=dtype)[:, :k].copy_(x)
    gain = (1 + 0.3 * torch.randn(k, device="cuda", generator=g)).to(dtype)
    check_norm(hq.f8_rmsnorm(wide, gain, 1e-5, values=True), wide, gain, 1e-5, None)


@pytest.mark.parametrize("eps", [1e30, 1e36, 3e38])
def test_a_large_epsilon_counts(hq, eps):
    """Its mean square is no smaller than the row's, whose sum of squares passes fp32."""
    x = torch.full((2, 32768), 1e18, device="cuda")
    x[1, ::2] = 3e17
    gain = torch.ones(32768, device="cuda")
    check_norm(hq.f8_rmsnorm(x, gain, eps, values=True), x, gain, torch.tensor(eps, dtype=torch.float32).item(), None)
    one = torch.full((1, 8), 1.5e19, device="cuda")[:, :1]               # its square and eps are fp32 numbers, their sum is not always one
    check_norm(hq.f8_rmsnorm(one, gain[:1], eps, values=True), one, gain[:1], torch.tensor(eps, dtype=torch.float32).item(), None)
