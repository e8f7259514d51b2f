"""Serving calls one behind the other on buffers that are used again: each reads what the call before has written, although its CTAs may be
up before that call ends."""
import pytest
import torch

from gpu_util import hq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 3, 8, 12, 40])
def test_layers_read_what_the_call_before_wrote(hq, rows):
    g = torch.Generator("cuda").manual_seed(rows)
    k, steps = 512, 60

    def layer(n, k):
        codes = torch.randint(0, 256, (n, k // 2), device="cuda", dtype=torch.uint8, generator=g)
        return hq.linear_create(codes, (torch.rand(n, k // 64, device="cuda", generator=g) / k).bfloat16(), k, 64)

    down, up, cache = layer(k, k), layer(k, k), hq.kv_cache(rows * 4, 2, 16, 64)
    for t in (cache.k, cache.v):
        t.random_(-127, 128, generator=g)
    for t in (cache.k_scale, cache.v_scale):
        t.uniform_(0.01, 0.03, generator=g)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    starts, lens, table = ints(range(rows + 1)), ints([10 + 5 * (r % 10) for r in range(rows)]), ints(range(rows * 4)).view(rows, 4)
    x = torch.randn(steps, rows, k, device="cuda", generator=g).bfloat16()
    a, b, c, d = (torch.empty(rows, k, dtype=torch.bfloat16, device="cuda") for _ in range(4))

    def run(stop):
        out = []
        for i in range(steps):
            for call in (lambda: down(x[i], out=a), lambda: cache.attention(a.view(rows, 8, 64), starts, lens, table, out=b.view(rows, 8, 64)),
                         lambda: up(b, out=c), lambda: down(c, out=d)):
                call()
                if stop:
                    torch.cuda.synchronize()
            out.append(d.clone())
        return torch.stack(out)

    want = run(True)
    assert len(want.flatten(1).unique(dim=0)) == steps
    for _ in range(5):
        assert torch.equal(run(False), want)
