"""Admission, quantizing append and read-back of the 8-bit key/value cache: whole numbers, codes and scales equal the
oracle's exactly (both sides take the same IEEE fp32 steps)."""
import numpy as np
import pytest
import torch

from gpu_util import hq  # noqa: F401
from oracle import serving
from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu


def ints(v, dtype=torch.int32):
    return torch.tensor(np.asarray(v), dtype=dtype).cuda()


# ---- admission ------------------------------------------------------------------------------------------------
def admission(seed, requests, cached_max, added_max, block, spare=3):
    g = np.random.default_rng(seed)
    cached, added = g.integers(0, cached_max + 1, requests), g.integers(0, added_max + 1, requests)
    width = -(-int((cached + added).max()) // block) + 1
    have = -(-cached // block)
    need = int((-(-(cached + added) // block) - have).sum())
    ids = g.permutation(int(have.sum()) + need + spare).astype(np.int32)
    table = np.full((requests, width), -7, np.int32)
    at = 0
    for r in range(requests):
        table[r, :have[r]] = ids[at:at + have[r]]
        at += have[r]
    return cached, added, table, ids[at:], need


def run_schedule(hq, cached, added, table, free, block, capacity):
    t = ints(table)
    out = hq.kv_schedule(ints(cached), ints(added), t, ints(free) if len(free) else ints([0]), ints([len(free)]), block, capacity)
    return [t.cpu().numpy()] + [o.cpu().numpy() for o in out]


@pytest.mark.parametrize("requests,cached_max,added_max,block", [
    (1, 0, 1, 16), (1, 100, 0, 16), (2, 40, 40, 32), (31, 500, 1, 16), (33, 5, 5, 1), (97, 1000, 1, 32), (512, 300, 3, 16), (513, 64, 200, 64),
    (1501, 100, 30, 16), (8192, 20, 4, 16), (3, 0, 20000, 128), (7, 50, 9, 48)])
def test_schedule_matches_oracle(hq, requests, cached_max, added_max, block):
    for seed in (1, 2):
        cached, added, table, free, need = admission(seed, requests, cached_max, added_max, block)
        for capacity in (int(added.sum()), int(added.sum()) + 13):
            got = run_schedule(hq, cached, added, table, free, block, capacity)
            want = serving.schedule(cached, added, table, list(free), block, capacity)
            for a, b in zip(got, want):
                assert np.array_equal(a, b)
        exact = free[len(free) - need:]                                  # not one block to spare
        got = run_schedule(hq, cached, added, table, exact, block, int(added.sum()))
        assert got[4].tolist() == [0, int(added.sum()), need, 0]


def test_schedule_refuses_all_or_nothing(hq):
    cached, added, table, free, need = admission(5, 40, 100, 30, 16)
    assert need > 1
    neg = added.copy()
    neg[7] = -1
    negc = cached.copy()
    negc[39] = -5
    for c, m, tab, fr, cap in ((cached, added, table, free[:need - 1], 2000), (cached, added, table[:, :2], free, 2000),
                               (cached, added, table, free, int(added.sum()) - 1), (cached, neg, table, free, 2000), (negc, added, table, free, 2000),
                               (cached, added, table, free[:0], 2000)):
        got = run_schedule(hq, c, m, np.ascontiguousarray(tab), fr, 16, cap)
        want = serving.schedule(c, m, tab, list(fr), 16, cap)
        assert want[4][3] == 1
        for a, b in zip(got, want):
            assert np.array_equal(a, b)


def test_schedule_lengths_whose_sum_passes_32_bits(hq):
    big = 2 ** 31 - 1
    got = run_schedule(hq, [big, big, 3], [0, 0, 1], np.zeros((3, 4), np.int32), [1, 2], 16, 8)
    assert got[4].tolist() == [2, 0, 0, 1] and got[2].tolist() == [big, big, 3]
    got = run_schedule(hq, [0, 0], [big, big], np.zeros((2, 4), np.int32), [1, 2], 16, 8)
    assert got[4].tolist() == [2, 0, 0, 1] and set(got[3].tolist()) == {-1}


def test_schedule_argument_refusals(hq):
    a = ints([1])
    with pytest.raises(qtz.QtzError) as e:
        hq.kv_schedule(ints(np.zeros(8193)), ints(np.zeros(8193)), ints(np.zeros((8193, 1))), a, a, 16, 1)
    assert e.value.code == -9
    with pytest.raises(qtz.QtzError) as e:
        hq.kv_schedule(a, a, ints([[0]]), a, a, 0, 1)
    assert e.value.code == -1
    with pytest.raises(ValueError):
        hq.kv_schedule(a, ints([1, 2]), ints([[0]]), a, a, 16, 1)
    with pytest.raises(ValueError):
        hq.kv_schedule(a.long(), a, ints([[0]]), a, a, 16, 1)


# ---- append and read --------------------------------------------------------------------------------------------
def random_cache(hq, g, blocks, heads, block, dim):
    codes = [g.integers(-127, 128, (blocks, heads, block, dim)).astype(np.int8) for _ in range(2)]
    scales = [g.uniform(0.005, 0.05, (blocks, heads)).astype(np.float32) for _ in range(2)]
    cache = qtz.KvCache(hq, *(torch.from_numpy(c.copy()).cuda() for c in codes), *(torch.from_numpy(s.copy()).cuda() for s in scales))
    return cache, codes, scales


def values(g, dtype, tokens, heads, dim):
    """Keys and values as slices of one projection: strided, and some heads much larger than others."""
    x = torch.from_numpy(g.normal(size=(tokens, 4 * heads, dim)).astype(np.float32) * g.choice([0.01, 1.0, 30.0], (tokens, 4 * heads, 1)).astype(np.float32))
    x = x.to(dtype).cuda()
    return x[:, heads:2 * heads], x[:, 3 * heads:]


def check_append(cache, codes, scales, k, v, slots, written=None):
    cache.append(k, v, ints(slots, torch.int64))
    got = [(cache.k, cache.k_scale), (cache.v, cache.v_scale)]
    out = []
    for x, c, s, (gc, gs) in zip((k, v), codes, scales, got):
        wc, ws = serving.append(c, s, x.float().cpu().numpy(), slots)
        assert np.array_equal(gs.cpu().numpy(), ws)
        assert np.array_equal(gc.cpu().numpy(), wc)
        out.append((wc, ws))
    return [c for c, _ in out], [s for _, s in out]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,dim,block", [(1, 64, 16), (3, 128, 32), (2, 256, 16), (8, 64, 128), (2, 128, 256), (5, 128, 48)])
def test_append_matches_oracle_bit_for_bit(hq, heads, dim, block, dtype):
    g = np.random.default_rng(heads * dim + block)
    cache, codes, scales = random_cache(hq, g, 11, heads, block, dim)
    order = g.permutation(11)
    run = lambda b, lo, hi: [int(order[b]) * block + o for o in range(lo, hi)]  # noqa: E731
    # a single token at every kind of place, a partly filled block, whole blocks, the join of two, skipped entries
    steps = [run(0, 0, 1), run(0, 1, 2), run(1, 3, 4) + run(2, block - 1, block) + run(3, 0, 1), run(0, 2, block), run(4, 5, block) + run(5, 0, block) + run(6, 0, 7),
             [-1] + run(7, 0, 3) + [-1, -1] + run(8, 2, 3) + [-1], [-1, -1], run(0, 0, block) + run(7, 3, 4)]
    for slots in steps:
        k, v = values(g, dtype, len(slots), heads, dim)
        codes, scales = check_append(cache, codes, scales, k, v, slots)


def test_append_of_many_tokens(hq):
    g = np.random.default_rng(77)
    heads, dim, block = 4, 128, 64
    cache, codes, scales = random_cache(hq, g, 40, heads, block, dim)
    order = g.permutation(40)
    slots = [int(order[i // block]) * block + i % block for i in range(13, 39 * block + 5)]
    k, v = values(g, torch.bfloat16, len(slots), heads, dim)
    codes, scales = check_append(cache, codes, scales, k, v, slots)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_append_of_runs_on_either_side_of_what_a_warp_takes(hq, dim):
    """A lane holds 4 pieces of 8 values and its warp takes 8 at most: runs one token shorter and longer than both, at offset 0 and
    behind older tokens, side by side."""
    g = np.random.default_rng(79 + dim)
    heads, block, most = 2, 64, 256 * 8 // dim
    lens = [most // 2 - 1, most // 2, most // 2 + 1, most - 1, most, most + 1]
    cache, codes, scales = random_cache(hq, g, 12, heads, block, dim)
    order = g.permutation(12)
    slots = [int(order[2 * i + at]) * block + o for i, n in enumerate(lens) for at, lo in ((0, 0), (1, 3)) for o in range(lo, lo + n)]
    for _ in range(2):
        k, v = values(g, torch.float16, len(slots), heads, dim)
        codes, scales = check_append(cache, codes, scales, k, v, slots)


def test_append_of_values_that_are_hard(hq):
    """Zeros, infinities, NaN, the smallest and the largest values, exact ties of the rounding."""
    g = np.random.default_rng(78)
    for dtype in (torch.float16, torch.bfloat16):
        cache, codes, scales = random_cache(hq, g, 8, 2, 16, 64)
        big = torch.finfo(dtype).max
        rows = [torch.zeros(64), torch.full((64,), float("nan")), torch.cat((torch.full((32,), float("inf")), torch.ones(32))),
                torch.full((64,), 2.0 ** -24), torch.full((64,), big), torch.linspace(-127, 127, 64).round() / 2, torch.full((64,), -float("inf"))]
        for i, row in enumerate(rows):
            x = row.to(dtype).expand(1, 2, 64).contiguous().cuda()
            codes, scales = check_append(cache, codes, scales, x, x * 2, [i * 16])
            codes, scales = check_append(cache, codes, scales, x * 0.75, x, [i * 16 + 1])
        assert np.isfinite(scales[0]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,dim,block", [(1, 64, 16), (3, 128, 32), (2, 256, 64)])
def test_read_matches_oracle(hq, heads, dim, block, dtype):
    g = np.random.default_rng(80)
    cache, codes, scales = random_cache(hq, g, 9, heads, block, dim)
    cache.k_scale[3] = 0.0                                                   # counts as 2^-100
    scales[0][3] = 0.0
    for count in (1, 2, 37, 400):
        slots = g.integers(-2, 9 * block, count)
        slots[0] = 3 * block if count > 1 else slots[0]
        k, v = cache.read(ints(slots, torch.int64), dtype=dtype)
        for got, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
            want = torch.from_numpy(serving.read(c, s, slots)).to(dtype)
            assert torch.equal(got.cpu(), want)
    assert cache.read(ints([], torch.int64), dtype=dtype)[0].shape == (0, heads, dim)


def test_slots_outside_the_cache_are_skipped_and_reported(hq):
    g = np.random.default_rng(81)
    cache, codes, scales = random_cache(hq, g, 4, 2, 16, 64)
    slots = [5, 4 * 16, 10 ** 12]
    k, v = values(g, torch.bfloat16, 3, 2, 64)
    cache.append(k, v, ints(slots, torch.int64))
    assert hq.device_status() == (-1, 10)
    want, _ = serving.append(codes[0], scales[0], k.float().cpu().numpy(), [5, -1, -1])
    assert np.array_equal(cache.k.cpu().numpy(), want)
    got, _ = cache.read(ints([5, 64, -3], torch.int64))
    assert hq.device_status() == (-1, 11) and not got[1:].any() and got[0].any()
    assert hq.device_status()[0] == 0


def test_append_and_read_on_another_stream(hq):
    g = np.random.default_rng(82)
    cache, codes, scales = random_cache(hq, g, 4, 2, 16, 128)
    k, v = values(g, torch.float16, 20, 2, 128)
    slots = list(range(16, 36))
    side = torch.cuda.Stream()
    s = ints(slots, torch.int64)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.append(k, v, s)
        got, _ = cache.read(s)
    side.synchronize()
    wc, ws = serving.append(codes[0], scales[0], k.float().cpu().numpy(), slots)
    assert np.array_equal(got.cpu().numpy(), serving.read(wc, ws, slots))


def test_refusals(hq):
    cache = hq.kv_cache(2, 2, 16, 64)
    k = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    s = ints([0], torch.int64)
    for shape, code in (((2, 2, 16, 96), -3), ((2, 2, 24, 64), -3), ((2, 2, 512, 64), -3)):
        c = hq.kv_cache(*shape)
        with pytest.raises(qtz.QtzError) as e:
            c.append(torch.zeros(1, 2, shape[3], dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 2, shape[3], dtype=torch.bfloat16, device="cuda"), s)
        assert e.value.code == code
    with pytest.raises(qtz.QtzError) as e:
        cache.append(k.float(), k.float(), s)
    assert e.value.code == -1
    with pytest.raises(ValueError):
        cache.append(k, k[:, :1], s)
    with pytest.raises(ValueError):
        cache.append(k, k, s.int())
    odd = torch.zeros(1 * 2 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(qtz.QtzError) as e:
        cache.append(odd[1:129].view(1, 2, 64), k, s)
    assert e.value.code == -2
    with pytest.raises(qtz.QtzError) as e:
        cache.append(odd.as_strided((1, 2, 64), (132, 66, 1)), k, s)
    assert e.value.code == -2
    with pytest.raises(qtz.QtzError) as e:
        cache.read(s, dtype=torch.float64)
    assert e.value.code == -1
    with pytest.raises(ValueError):
        qtz.KvCache(hq, cache.k, cache.v[:1], cache.k_scale, cache.v_scale)
    lib = qtz.load_library()
    assert lib.qtz_kv_append(None, cache._ref, k.data_ptr(), 128, 64, k.data_ptr(), 128, 64, 18, s.data_ptr(), 1, None) == -1
    assert lib.qtz_kv_append(hq.h, cache._ref, k.data_ptr(), 128, 64, k.data_ptr(), 128, 64, 18, s.data_ptr(), -1, None) == -1
    assert lib.qtz_kv_append(hq.h, cache._ref, None, 128, 64, k.data_ptr(), 128, 64, 18, s.data_ptr(), 1, None) == -1
    assert lib.qtz_kv_read(hq.h, None, s.data_ptr(), 1, 16, k.data_ptr(), k.data_ptr(), None) == -1
