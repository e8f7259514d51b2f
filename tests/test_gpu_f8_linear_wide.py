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


@pytest.mark.parametrize("rows,n,k", [(300, 77, 100), (2305, 2087, 260), (4999, 1288, 128), (1290, 5003, 640), (250, 10007, 2100), (131, 13001, 1930), (300, 10303, 2050)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("pad", [0, 16])
def test_whole_tiles_leave_what_lies_beside_y(hq, rows, n, k, dtype, pad):
    """Pairs with a tile or several each; rows of y that start on 16 bytes and end anywhere, and rows that do not."""
    x, xs, w, ws, bias = make(rows, n, k, n)
    plan = hq.f8_linear_create(w, ws, bias=bias)
    around = torch.full((rows + 2, -(-n // 8) * 8 + pad + (0 if pad else 1)), 7.0, device="cuda", dtype=dtype)
    y = around[1:-1, pad // 2:pad // 2 + n]
    plan(x, xs, out=y)
    check(y, x, xs, w, ws, bias, rows=[r for r in (0, 31, 127, 128, 255, 256, rows // 2, rows - 2, rows - 1) if r < rows])
    few = torch.cat([plan(x[r:r + 100], xs[r:r + 100], dtype=dtype) for r in range(0, rows, 100)])
    off = (y.double() - few.double()).abs()
    assert bool((off <= 2.0 ** -7 * few.double().abs() + 1e-3 * few.double().abs().max()).all())   # every row is in its place
    y.fill_(7)
    assert bool((around == 7).all())                                            # nothing beside y was written
    assert hq.device_status() == (0, 0)
