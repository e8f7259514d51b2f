"""Plans and caches whose handle is closed before them."""
import pytest
import torch

from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu


def test_plans_and_caches_outlive_their_handle_and_refuse_calls():
    kept = qtz.Handle(0)
    codes = torch.full((32, 32), 0x21, dtype=torch.uint8, device="cuda")
    scales, x = torch.ones(32, 1, dtype=torch.bfloat16, device="cuda"), torch.ones(1, 64, dtype=torch.bfloat16, device="cuda")
    other = kept.linear_create(codes, scales, 64, 64)
    want = other(x)
    assert bool((want == 96).all())                                    # 32 (1 + 2)
    for _ in range(20):
        h = qtz.Handle(0)
        plan, cache = h.linear_create(codes, scales, 64, 64), h.kv_cache(1, 1, 16, 64)
        h.close()
        with pytest.raises(ValueError):
            plan(x)
        slot, row = torch.zeros(1, dtype=torch.int64, device="cuda"), x.view(1, 1, 64)
        ints = torch.zeros(2, dtype=torch.int32, device="cuda")
        for call in (lambda: cache.append(row, row, slot), lambda: cache.read(slot), lambda: cache.attention(row, ints, ints[:1], ints[:1].view(1, 1))):
            with pytest.raises(qtz.QtzError) as e:
                call()
            assert e.value.code == -1
        plan.close()
        assert torch.equal(other(x), want)
    kept.close()
    other.close()
