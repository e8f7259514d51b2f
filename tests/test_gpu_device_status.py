"""What device code records and the host reads: neither kind of report hides the other."""
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
