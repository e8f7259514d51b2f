"""Wide layers, many rows and every way of splitting the work of the 8-bit floating-point linear layers, against fp64."""
import pytest
import torch

from gpu_util import hq  # noqa: F401
from paper_1806_08342_b200 import qtz
from test_gpu_f8_linear import check, make

pytestmark = pytest.mark.gpu

# more tiles than SMs with few and many rows; several tiles a pair; clusters of every size that splits columns
CASES = [(5, 38100, 260), (33, 40001, 130), (100, 38000, 257), (129, 20000, 130), (300, 19000, 300), (700, 30000, 128), (2500, 9000, 300),
         (1, 256, 1920), (1, 512, 8192), (3, 4000, 700), (20, 1300, 1150), (70, 800, 2900), (128, 2100, 640), (130, 256, 2048), (250, 700, 1100), (260, 300, 4000),
         (600, 1025, 1500), (1100, 4097, 520)]


@pytest.mark.parametrize("case", CASES)
def test_every_split(hq, case):
    rows, n, k = case
    x, xs, w, ws, bias = make(rows, n, k, 7 * rows + n)
    plan = hq.f8_linear_create(w, ws, bias=bias)
    y = plan(x, xs, dtype=torch.float32)
    pick = torch.arange(rows) if rows <= 40 else torch.cat([torch.arange(3), torch.randint(0, rows, (20,), generator=torch.Generator().manual_seed(n)), torch.arange(rows - 3, rows)])
    check(y, x, xs, w, ws, bias, rows=pick.cuda())
    full = torch.empty_like(y)
    full.fill_(float("nan"))
    assert torch.equal(plan(x, xs, out=full), y) and bool(torch.isfinite(full).all())       # every value is written, the same when repeated
    plan.close()


def test_values_and_rows_beyond_32_bits(hq):
    """70001 x 33000 values of y: the first rows, some at the crossing, the last ones."""
    rows, n, k = 70001, 33000, 128
    _, _, w, ws, bias = make(1, n, k, 5)
    x, xs, *_ = make(rows, 1, k, 6)
    y = hq.f8_linear_create(w, ws, bias=bias)(x, xs)
    cross = 2 ** 31 // n
    check(y, x, xs, w, ws, bias, rows=torch.tensor([0, 1, cross - 1, cross, cross + 1, rows - 2, rows - 1], device="cuda"))
    torch.cuda.empty_cache()


def test_codes_beyond_32_bits(hq):
    """Rows of x that lie past 2^32 bytes."""
    rows, k = 300, 384
    _, _, w, ws, _ = make(1, 200, k, 8)
    pitch = 16 << 20
    x = torch.zeros(rows * pitch, device="cuda", dtype=torch.uint8).view(rows, pitch)[:, :k]
    small, xs, *_ = make(rows, 1, k, 9)
    x.copy_(small.view(torch.uint8))
    plan = hq.f8_linear_create(w, ws)
    assert torch.equal(plan(x.view(qtz.E4M3), xs), plan(small, xs))
    torch.cuda.empty_cache()
