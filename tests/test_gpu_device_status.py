"""What device code records and the host reads: neither kind of report hides the other, and what a caller does after a timeout."""
import pytest
import torch

from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu


@pytest.fixture
def handle():
    h = qtz.Handle(0)
    yield h
    h.close()


def test_a_timeout_is_reported_over_an_id_outside_the_cache(handle):
    """An unread report of a skipped slot must not hide that later results are void."""
    cache = handle.kv_cache(2, 1, 16, 64)
    x = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    outside = torch.tensor([1000], device="cuda")
    cache.append(x, x, outside)
    handle.selftest_wait_timeout(20000)
    assert handle.device_status() == (-7, 8)
    assert handle.device_status() == (-1, 10)                          # then the skipped slot
    assert handle.device_status() == (0, 0)
    handle.selftest_wait_timeout(20000)
    cache.append(x, x, outside)
    assert handle.device_status() == (-7, 8)
    cache.read(outside)                                                # the first of the skipped ones is kept
    assert handle.device_status() == (-1, 10)
    assert handle.device_status() == (0, 0)


def test_attention_after_a_reported_timeout(handle):
    """A call that gave up leaves parts counted in the workspace of its cache: reporting the timeout makes it ready again."""
    g = torch.Generator("cuda").manual_seed(3)
    cache = handle.kv_cache(600, 1, 16, 64)
    cache.k.random_(-127, 128, generator=g)
    cache.v.random_(-127, 128, generator=g)
    cache.k_scale.fill_(0.02)
    cache.v_scale.fill_(0.02)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.randn(1, 4, 64, device="cuda", generator=g).bfloat16()
    call = lambda: cache.attention(q, ints(0, 1), ints(9000), torch.arange(600, dtype=torch.int32, device="cuda")[None])  # noqa: E731
    want = call()
    assert bool(want.any())
    cache.workspace.fill_(1)                                           # as a call would leave it that gave up on the way
    handle.selftest_wait_timeout(20000)
    assert handle.device_status() == (-7, 8)
    assert torch.equal(call(), want)
    cache.workspace.fill_(1)
    cache.reset_workspace()
    assert torch.equal(call(), want)
