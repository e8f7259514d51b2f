"""8-bit floating-point linear layers whose waits run out, with other calls straight behind them: those start on the same SMs, in the
shared and tensor memory that the layers leave.  The scales of the activations lie in pinned host memory, each in a place of its own, so
that a block's scales arrive long after its loads and the waits for them outlast the least budget."""
import time

import pytest
import torch

from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu

LEAST, USUAL = 1000, 2_000_000_000
CASES = [  # rows, n, k: single CTAs whose columns are shared (three) or not, pairs that share columns, pairs with a tile or several, of either width
    (1, 4096, 8192), (30, 5000, 2048), (200, 2000, 8192), (128, 40000, 2048), (1000, 1000, 8192), (1000, 4096, 4096), (2500, 9000, 4000),
    (777, 6144, 4096)]


def layer(h, rows, n, k, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    plan = h.f8_linear_create(*h.f8_quantize_weights(torch.randn(n, k, device="cuda", generator=g)))
    codes, scales = h.f8_quantize(torch.randn(rows, k, device="cuda", generator=g))
    return plan, codes, scales


@pytest.mark.parametrize("case", CASES)
def test_calls_straight_behind_one_whose_waits_run_out(case):
    h, other = qtz.Handle(0), qtz.Handle(0)
    plan, codes, scales = layer(h, *case, 1)
    rows, blocks = scales.shape
    far = torch.zeros(rows, blocks, 16).pin_memory()
    far[:, :, 0] = scales.cpu()
    out = torch.empty(rows, plan.n, device="cuda", dtype=torch.bfloat16)
    want = plan(codes, scales)
    next_calls = [layer(other, *sizes, 2) for sizes in ((3, 38000, 300), (600, 5000, 512), (300, 1000, 4096))]
    next_want = [p(*x) for p, *x in next_calls]
    assert h.device_status() == (0, 0)

    def slow():
        assert plan._run(plan.plan, codes.data_ptr(), codes.stride(0), far.data_ptr(), blocks * 16, 16, rows, out.data_ptr(), plan.n, qtz.BF16,
                         torch.cuda.current_stream().cuda_stream) == 0

    slow()
    assert h.device_status() == (0, 0) and torch.equal(out, want)
    ran_out = 0
    for turn in range(6):
        h.set_wait_budget(LEAST)
        begin = time.perf_counter()
        slow()
        h.set_wait_budget(USUAL)
        p, *x = next_calls[turn % 3]
        behind = p(*x)
        torch.cuda.synchronize()
        assert time.perf_counter() - begin < 0.5                         # a wait for what does not come would take a second
        status = h.device_status()
        assert status == (-7, 14) or (status == (0, 0) and torch.equal(out, want))
        ran_out += status != (0, 0)
        assert torch.equal(behind, next_want[turn % 3]) and other.device_status() == (0, 0)
        slow()
        assert torch.equal(out, want) and torch.equal(plan(codes, scales), want) and h.device_status() == (0, 0)
    assert ran_out > 0 or rows < 100                                     # few rows' scales may arrive within the polls that a wait always makes
    h.close()
    other.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n,k", [(777, 6144, 4096), (777, 6144, 2048), (1500, 4608, 2100)])
def test_rows_on_their_way_are_not_overtaken_by_the_next_tile(rows, n, k, dtype):
    """Pairs with several tiles of 192 columns: 96 columns of 16 bits leave in three steps through two places.  The sums are those of the
    call in 32 bits, while the memory is busy with copies."""
    h = qtz.Handle(0)
    plan, codes, scales = layer(h, rows, n, k, 3)
    want = plan(codes, scales, dtype=torch.float32).to(dtype)
    busy, side = torch.empty(2, 128 << 20, device="cuda"), torch.cuda.Stream()
    for _ in range(10):
        with torch.cuda.stream(side):
            busy[0].copy_(busy[1])
        assert torch.equal(plan(codes, scales, dtype=dtype), want)
    assert h.device_status() == (0, 0)
    h.close()
