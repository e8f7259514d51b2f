"""How the attention over the 8-bit cache is called: captures, stored scales, wide tables, strides of single rows."""
import numpy as np
import pytest
import torch

from gpu_util import hq  # noqa: F401
from oracle import serving
from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu


def ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def make(hq, seed, lens, added, kv_heads, group, dim, block, dtype=torch.bfloat16):
    """(cache, codes, scales, q, starts, lens, table) with everything on the device but codes and scales."""
    g = np.random.default_rng(seed)
    need = [-(-v // block) for v in lens]
    blocks = sum(need) + 1
    codes = [g.integers(-127, 128, (blocks, kv_heads, block, dim)).astype(np.int8) for _ in range(2)]
    scales = [g.uniform(0.005, 0.03, (blocks, kv_heads)).astype(np.float32) for _ in range(2)]
    table, at = np.zeros((len(lens), max(need)), np.int32), 0
    for r, n in enumerate(need):
        table[r, :n] = np.arange(at, at + n)
        at += n
    starts = np.concatenate(([0], np.cumsum(added)))
    q = torch.from_numpy(g.normal(size=(int(starts[-1]), kv_heads * group, dim))).to(dtype)
    cache = qtz.KvCache(hq, *(torch.from_numpy(c).cuda() for c in codes), *(torch.from_numpy(s).cuda() for s in scales))
    return cache, codes, scales, q.cuda(), ints(starts.tolist()), ints(lens), torch.from_numpy(table).cuda()


def test_first_call_of_a_cache_inside_a_capture(hq):
    """What a call needs is there before it is captured: a plain call before the first replay gives the same as after it, even if the
    memory that the capture is given holds something."""
    cache, codes, scales, q, starts, lens, table = make(hq, 1, [9000, 4100], [1, 1], 2, 4, 128, 32)
    want = qtz.KvCache(hq, cache.k, cache.v, cache.k_scale, cache.v_scale).attention(q, starts, lens, table)
    pool, junk, graph, out = torch.cuda.graph_pool_handle(), torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(junk, pool=pool):
        held = [torch.full((8 << 20,), 77, dtype=torch.int32, device="cuda") for _ in range(2)]
    junk.replay()
    torch.cuda.synchronize()
    del held                                                                # the pool hands this memory out again
    with torch.cuda.graph(graph, pool=pool):
        cache.attention(q, starts, lens, table, out=out)
    for _ in range(3):
        assert torch.equal(cache.attention(q, starts, lens, table), want)
    for _ in range(2):
        graph.replay()
        assert torch.equal(out, want)
        assert torch.equal(cache.attention(q, starts, lens, table), want)


def test_stored_scales_below_the_least_one_count_as_it(hq):
    """Zero, negative and NaN scales, which append never writes, count as 2^-100 in either tensor, as in the read-back."""
    for at, value in ((0, -0.02), (1, -1e30), (0, 0.0), (1, 0.0), (0, -float("inf")), (0, float("nan"))):
        cache, codes, scales, q, starts, lens, table = make(hq, 2, [200, 64], [1, 2], 2, 2, 64, 16)
        (cache.k_scale, cache.v_scale)[at][1::2] = value
        scales[at][1::2] = 2.0 ** -100
        y, lse = cache.attention(q, starts, lens, table, return_lse=True)
        want, want_lse = serving.attention(q.double().cpu().numpy(), codes[0], scales[0], codes[1], scales[1], starts.tolist(), lens.tolist(),
                                           table.cpu().numpy(), 64 ** -0.5)
        assert np.allclose(lse.double().cpu().numpy(), want_lse, rtol=0, atol=2e-4), (at, value)
        assert np.allclose(y.double().cpu().numpy(), want, rtol=2.0 ** -8, atol=2e-3), (at, value)


def test_strides_of_single_rows_and_heads_do_not_matter(hq):
    """An axis of one element has no stride: a row of a matrix of odd pitch, one head of a single-head cache."""
    cache, codes, scales, q, starts, lens, table = make(hq, 4, [100], [1], 1, 4, 64, 16)
    want = cache.attention(q, starts, lens, table)
    row = lambda t: torch.zeros(1024, dtype=q.dtype, device="cuda").as_strided((1, 4, 64), (261, 64, 1)).copy_(t)  # noqa: E731
    assert torch.equal(cache.attention(row(q), starts, lens, table, out=row(want)), want)
    cache, codes, scales, q, starts, lens, table = make(hq, 5, [100, 50], [1, 1], 1, 1, 64, 16)
    want = cache.attention(q, starts, lens, table)
    head = lambda t: torch.zeros(1024, dtype=q.dtype, device="cuda").as_strided((2, 1, 64), (64, 77, 1)).copy_(t)  # noqa: E731
    assert torch.equal(cache.attention(head(q), starts, lens, table, out=head(want)), want)
    got, same = hq.kv_cache(2, 1, 16, 64), hq.kv_cache(2, 1, 16, 64)
    for c, k in ((got, head(q)), (same, q)):
        c.append(k, k, ints([3, 4], torch.int64))
        c.append(k[:1].as_strided((1, 1, 64), (13, 13, 1)), k[:1], ints([5], torch.int64))
    assert torch.equal(got.k, same.k) and torch.equal(got.v_scale, same.v_scale) and bool(same.k.any())


def test_many_rows_beside_a_wide_table(hq):
    """A long step on a table for long requests: what counts is the lengths, and most of these rows are padding."""
    cache, codes, scales, q, starts, lens, table = make(hq, 3, [300, 20], [30, 20], 8, 8, 64, 256)
    wide = torch.zeros(2, 1024, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    many = torch.zeros(65536, 64, 64, dtype=q.dtype, device="cuda")
    many[:50] = q
    y, out = cache.attention(q, starts, lens, table), torch.full_like(many, 3.0)
    cache.attention(many, starts, lens, wide, out=out)
    assert torch.allclose(out[:50].float(), y.float(), rtol=2.0 ** -7, atol=1e-5) and bool((out[50:] == 3.0).all())
