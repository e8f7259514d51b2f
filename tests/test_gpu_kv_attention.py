"""Attention over the 8-bit cache through the public entry points against fp64.

Bound of a row, with c = softmax scale, p the exact probabilities, u the output type's half unit:
  logits   products of a query and a code are exact; sums over the head, scaling and the queries' common exponent cost
           d_l = 2 (D + 8) 2^-24 c max_p sum |q k| + D 2^-24 c max|q| max|k|
  weights  relative: d_l twice (numerator and sum), 2^-11 for their rounding to fp16, 2^-18 for exponentials and scales
  y        (2 d_l + 2^-10 + 2^-18) sum p |v| + 2^-24 max|v| + u |y|
  lse      d_l + 2^-18 (1 + |lse|)"""
import numpy as np
import pytest
import torch

from gpu_util import hq  # noqa: F401
from oracle import serving
from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu

UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float16, torch.bfloat16)}


def setup(hq, seed, lens, added, kv_heads, group, dim, block, dtype, spare=2, k_scale=(0.005, 0.04), v_scale=(0.005, 0.04), width=None, q_size=1.0):
    g = np.random.default_rng(seed)
    need = [-(-v // block) for v in lens]
    blocks = sum(need) + spare
    codes = [g.integers(-127, 128, (blocks, kv_heads, block, dim)).astype(np.int8) for _ in range(2)]
    logs = lambda lo, hi: np.exp(g.uniform(np.log(lo), np.log(hi), (blocks, kv_heads))).astype(np.float32)  # noqa: E731
    scales = [logs(*k_scale), logs(*v_scale)]
    ids = g.permutation(blocks).astype(np.int32)
    table = np.full((len(lens), (max(need) if width is None else width) or 1), 2 ** 30, np.int32)   # entries past the length: never used
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    starts = np.concatenate(([0], np.cumsum(added))).astype(np.int32)
    q = torch.from_numpy(g.normal(size=(int(starts[-1]), kv_heads * group, dim)).astype(np.float32) * q_size).to(dtype)
    cache = qtz.KvCache(hq, *(torch.from_numpy(c).cuda() for c in codes), *(torch.from_numpy(s).cuda() for s in scales))
    return cache, codes, scales, table, starts, np.array(lens, np.int32), q


def tolerances(q, codes, scales, starts, lens, table, scale, window, y, unit):
    """(tol_y, tol_lse) by the bound of the module's docstring."""
    q = np.abs(q.astype(np.float64))
    tokens, heads, dim = q.shape
    kv_heads, block = codes[0].shape[1], codes[0].shape[2]
    ty, tl = np.zeros((tokens, heads, dim)), np.zeros((tokens, heads))
    mags = [np.abs(c.astype(np.float64)) for c in codes]
    for r in range(len(lens)):
        used = table[r][:-(-int(lens[r]) // block)]
        if not len(used):
            continue
        for g in range(kv_heads):
            k, v = ((m[used, g] * s[used, g].astype(np.float64)[:, None, None]).reshape(-1, dim)[:lens[r]] for m, s in zip(mags, scales))
            for h in range(g * (heads // kv_heads), (g + 1) * (heads // kv_heads)):
                for t in range(starts[r], starts[r + 1]):
                    d = abs(scale) * (2 * (dim + 8) * 2.0 ** -24 * (k @ q[t, h]).max() + dim * 2.0 ** -24 * q[t, h].max() * k.max())
                    tl[t, h] = d
                    ty[t, h] = 2 * d + 2.0 ** -10 + 2.0 ** -18
    # sum p |v| from the oracle itself, with |v| in the place of v
    py, lse = serving.attention(np.asarray(tolerances.q), codes[0], scales[0], np.abs(codes[1]), scales[1], starts, lens, table, scale, window)
    vmax = (mags[1].max(axis=(2, 3)) * scales[1]).max()
    with np.errstate(invalid="ignore"):
        tl = tl + 2.0 ** -18 * (1 + np.where(np.isinf(lse), 0, np.abs(lse)))
    ty = ty * py + 2.0 ** -24 * vmax
    return ty + unit * (np.abs(y) + ty) + 2.0 ** -25, tl


def check(hq, made, scale=None, window=0, q_view=None, out=None):
    cache, codes, scales, table, starts, lens, q = made
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    qd = q.cuda() if q_view is None else q_view
    y, lse = cache.attention(qd, dev(starts), dev(lens), dev(table), scale=scale, window=window, return_lse=True, out=out)
    c = scale if scale is not None else q.shape[2] ** -0.5
    qn = q.double().numpy()
    want, want_lse = serving.attention(qn, codes[0], scales[0], codes[1], scales[1], starts, lens, table, c, window)
    tolerances.q = qn
    ty, tl = tolerances(qn, codes, scales, starts, lens, table, c, window, want, UNIT[q.dtype])
    got, got_lse = y.double().cpu().numpy(), lse.double().cpu().numpy()
    n = int(starts[-1])
    empty = np.isneginf(want_lse[:n])
    assert np.array_equal(np.isneginf(got_lse[:n]), empty) and not got[:n][empty].any()
    bad = ~(np.abs(got[:n] - want[:n]) <= ty[:n])
    assert not bad.any(), (np.argwhere(bad)[:4], got[:n][bad][:4], want[:n][bad][:4], ty[:n][bad][:4])
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got_lse[:n] - want_lse[:n]) <= tl[:n]) & ~empty
    assert not bad.any(), (np.argwhere(bad)[:4], got_lse[:n][bad][:4], want_lse[:n][bad][:4])
    y2, lse2 = cache.attention(qd, dev(starts), dev(lens), dev(table), scale=scale, window=window, return_lse=True)
    assert torch.equal(y2[:n], y[:n]) and torch.equal(lse2[:n], lse[:n])                    # the same bits when repeated
    return y, lse


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,block,kv_heads,group", [(64, 16, 1, 1), (64, 32, 3, 5), (128, 16, 2, 4), (128, 48, 2, 8), (128, 64, 1, 16), (256, 32, 2, 3),
                                                     (256, 16, 1, 1), (128, 256, 4, 1), (64, 128, 1, 17)])
def test_attention_matches_fp64(hq, dim, block, kv_heads, group, dtype):
    lens = [1, 2, block - 1, block, block + 1, 0, 77, 3 * block + 5, 500]
    check(hq, setup(hq, dim + block + group, lens, [1] * len(lens), kv_heads, group, dim, block, dtype))


@pytest.mark.parametrize("added", [[1, 0, 3], [0, 0, 0, 7], [2, 5, 16, 33], [40]])
@pytest.mark.parametrize("window", [0, 1, 13, 64])
def test_several_new_tokens_and_windows(hq, added, window):
    lens = [a + (37 * i) % 90 for i, a in enumerate(added)]
    check(hq, setup(hq, sum(added) + window, lens, added, 2, 3, 64, 16, torch.bfloat16), window=window)
    check(hq, setup(hq, sum(added) + window + 1, lens, added, 1, 4, 128, 32, torch.float16), window=window)


def test_rows_that_see_nothing(hq):
    """Requests whose cache holds fewer tokens than they bring rows: the first rows lie before the cache."""
    made = setup(hq, 4, [3, 0, 1, 20], [5, 2, 1, 25], 2, 2, 64, 16, torch.bfloat16)
    _, lse = check(hq, made)
    assert torch.isneginf(lse).sum() == (2 + 2 + 0 + 5) * 4


@pytest.mark.parametrize("requests,length,kv_heads,group,dim", [(1, 20000, 1, 1, 64), (1, 9001, 2, 8, 128), (2, 7000, 1, 4, 256), (3, 4097, 4, 2, 128)])
def test_one_cache_split_over_many_blocks(hq, requests, length, kv_heads, group, dim):
    check(hq, setup(hq, length, [length - 13 * i for i in range(requests)], [1] * requests, kv_heads, group, dim, 64, torch.bfloat16))


def test_many_short_requests(hq):
    lens = [(7 * i) % 40 for i in range(700)]
    check(hq, setup(hq, 8, lens, [1] * 700, 1, 2, 64, 16, torch.float16))


def test_mixed_lengths_with_drafts_and_split(hq):
    lens = [9000, 12, 0, 700, 3, 2500]
    check(hq, setup(hq, 9, lens, [4, 1, 0, 9, 3, 20], 2, 4, 128, 32, torch.bfloat16))
    check(hq, setup(hq, 10, lens, [4, 1, 0, 9, 3, 20], 2, 4, 128, 32, torch.float16), window=300)


def test_large_logits_and_scales_far_apart(hq):
    """Softmax concentrated on few tokens; block scales over many orders of magnitude, the floor of 2^-100 among them."""
    made = setup(hq, 12, [300, 45], [1, 2], 2, 2, 64, 16, torch.float16, k_scale=(0.01, 1.0), q_size=2.0)
    check(hq, made)
    made = setup(hq, 13, [300, 45], [1, 2], 2, 2, 128, 16, torch.bfloat16, v_scale=(1e-12, 1e3))
    check(hq, made)
    made = setup(hq, 14, [200], [1], 1, 2, 64, 16, torch.bfloat16)
    made[0].v_scale[::2] = 2.0 ** -100
    made[2][1][::2] = 2.0 ** -100
    made[0].k_scale[1::3] = 2.0 ** -100
    made[2][0][1::3] = 2.0 ** -100
    check(hq, made)
    check(hq, setup(hq, 15, [90], [3], 1, 3, 64, 16, torch.bfloat16), scale=-0.3)
    check(hq, setup(hq, 16, [90], [3], 1, 3, 64, 16, torch.bfloat16), scale=0.0)


def test_queries_over_the_range_of_their_type(hq):
    """bf16 queries reach far beyond fp16: small and large rows, and rows whose elements differ by many orders."""
    cache, codes, scales, table, starts, lens, q = setup(hq, 17, [130, 70, 33, 50], [1] * 4, 1, 2, 128, 16, torch.bfloat16)
    q[0] *= 2.0 ** -60
    q[1] *= 2.0 ** 20
    cache.k_scale[table[1, :5]] *= 2.0 ** -20
    scales[0][table[1, :5]] *= np.float32(2.0 ** -20)
    q[2, :, ::2] *= 2.0 ** -30
    q[3] = 0
    check(hq, (cache, codes, scales, table, starts, lens, q))


def test_nan_in_a_query_stays_in_its_row(hq):
    cache, codes, scales, table, starts, lens, q = setup(hq, 18, [40, 40, 40], [1] * 3, 1, 4, 64, 16, torch.float16)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    clean, clean_lse = cache.attention(q.cuda(), dev(starts), dev(lens), dev(table), return_lse=True)
    q[1, 2, 5] = float("nan")
    y, lse = cache.attention(q.cuda(), dev(starts), dev(lens), dev(table), return_lse=True)
    assert torch.isnan(y[1, 2]).all() and torch.isnan(lse[1, 2])
    keep = torch.ones(3, 4, dtype=torch.bool)
    keep[1, 2] = False
    assert torch.equal(y.cpu()[keep], clean.cpu()[keep]) and torch.equal(lse.cpu()[keep], clean_lse.cpu()[keep])


def test_strides_padding_rows_and_streams(hq):
    made = setup(hq, 19, [100, 35], [2, 1], 2, 4, 64, 16, torch.bfloat16)
    cache, codes, scales, table, starts, lens, q = made
    fused = torch.full((5, 20, 64), float("nan"), dtype=torch.bfloat16, device="cuda")      # q heads 3 .. 10 of a projection; two rows of padding
    fused[:3, 3:11] = q.cuda()
    out = torch.full((5, 12, 64), 3.0, dtype=torch.bfloat16, device="cuda")[:, 2:10]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        check(hq, made, q_view=fused[:, 3:11], out=out)
    side.synchronize()
    assert (out[3:] == 3.0).all()
    whole = out._base
    assert (whole[:, :2] == 3.0).all() and (whole[:, 10:] == 3.0).all()


def test_requests_that_share_blocks(hq):
    cache, codes, scales, table, starts, lens, q = setup(hq, 20, [64, 64, 64], [1, 1, 1], 2, 2, 64, 16, torch.float16)
    table[1, :2] = table[0, :2]
    table[2] = table[0]
    check(hq, (cache, codes, scales, table, starts, lens, q))


def test_graph_replay_with_other_lengths(hq):
    """Lengths live on the device: a captured call follows them."""
    cache, codes, scales, table, starts, lens, q = setup(hq, 21, [600, 30], [1, 1], 2, 4, 128, 16, torch.bfloat16)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    qd, sd, ld, td = q.cuda(), dev(starts), dev(lens), dev(table)
    out = cache.attention(qd, sd, ld, td)                                                   # the first call makes the workspace
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attention(qd, sd, ld, td, out=out)
    for pair in ([600, 30], [5, 1], [0, 17], [577, 16]):
        ld.copy_(torch.tensor(pair, dtype=torch.int32))
        graph.replay()
        assert torch.equal(out, cache.attention(qd, sd, ld, td))
    want, _ = serving.attention(q.double().numpy(), codes[0], scales[0], codes[1], scales[1], starts, [577, 16], table, 128 ** -0.5)
    assert np.allclose(out.double().cpu().numpy(), want, rtol=2e-2, atol=2e-2)


def test_cache_whose_offsets_pass_32_bits(hq):
    blocks, heads, block, dim = 530_000, 2, 64, 64                                          # 4.34e9 codes each
    k = torch.empty(blocks, heads, block, dim, dtype=torch.int8, device="cuda")
    v = torch.empty_like(k)
    ks, vs = torch.empty(blocks, heads, device="cuda"), torch.empty(blocks, heads, device="cuda")
    made = setup(hq, 22, [150, 40], [1, 1], heads, 2, dim, block, torch.bfloat16, spare=0)
    small, codes, scales, table, starts, lens, q = made
    far = np.array([blocks - 1, 5, 262_144, 524_289], np.int32)                             # beyond 2^31 and 2^32 codes
    for i, b in enumerate(far):
        k[b], v[b], ks[b], vs[b] = small.k[i], small.v[i], small.k_scale[i], small.v_scale[i]
    cache = qtz.KvCache(hq, k, v, ks, vs)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    moved = far[np.minimum(table, 3)]
    y = cache.attention(q.cuda(), dev(starts), dev(lens), dev(moved))
    assert torch.equal(y, small.attention(q.cuda(), dev(starts), dev(lens), dev(table)))
    x = torch.randn(1, heads, dim, device="cuda").bfloat16()
    slot = torch.tensor([(blocks - 2) * block], device="cuda")
    cache.append(x, x, slot)
    got, _ = cache.read(slot)
    assert (got[0] - x[0].float()).abs().max() <= x.float().abs().max() / 127 * 0.51


def test_block_ids_outside_the_cache_are_reported(hq):
    cache, codes, scales, table, starts, lens, q = setup(hq, 23, [40, 40], [1, 1], 1, 2, 64, 16, torch.bfloat16)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    good = cache.attention(q.cuda(), dev(starts), dev(lens), dev(table))
    for wrong in (cache.blocks, -1, 2 ** 31 - 1):
        table[0, 1] = wrong
        y = cache.attention(q.cuda(), dev(starts), dev(lens), dev(table))
        assert hq.device_status() == (-1, 12)
        assert torch.equal(y[1], good[1]) and torch.isfinite(y).all()
    longer = dev(np.array([40, 41 + 16 * table.shape[1]], np.int32))                        # a length beyond its table is cut there
    table[0, 1] = 0
    y = cache.attention(q.cuda(), dev(starts), longer, dev(table))
    assert torch.isfinite(y).all()
    hq.device_status()


def test_refusals(hq):
    cache, codes, scales, table, starts, lens, q = setup(hq, 24, [20], [1], 2, 2, 64, 16, torch.bfloat16)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    qd, sd, ld, td = q.cuda(), dev(starts), dev(lens), dev(table)
    for args, code in (((qd[:, :3], sd, ld, td, None, 0), -1), ((qd, sd, ld, td, float("nan"), 0), -1), ((qd, sd, ld, td, None, -1), -1),
                       ((qd.float(), sd, ld, td, None, 0), -1)):
        with pytest.raises(qtz.QtzError) as e:
            cache.attention(*args)
        assert e.value.code == code
    odd = torch.zeros(4 * 66 + 8, dtype=torch.bfloat16, device="cuda")
    for view in (odd[1:257].view(1, 4, 64), odd[:264].view(1, 4, 66)[:, :, :64]):
        with pytest.raises(qtz.QtzError) as e:
            cache.attention(view, sd, ld, td)
        assert e.value.code == -2
    with pytest.raises(ValueError):
        cache.attention(qd, sd, ld.long(), td)
    with pytest.raises(ValueError):
        cache.attention(qd, ld, ld, td)
    with pytest.raises(ValueError):
        cache.attention(qd[:, :, :32], sd, ld, td)
    many = 8193
    with pytest.raises(qtz.QtzError) as e:
        cache.attention(qd, torch.zeros(many + 1, dtype=torch.int32, device="cuda"), torch.zeros(many, dtype=torch.int32, device="cuda"),
                        torch.zeros(many, 1, dtype=torch.int32, device="cuda"))
    assert e.value.code == -9
    lib = qtz.load_library()
    assert lib.qtz_kv_attention(hq.h, cache._ref, qd.data_ptr(), 256, 64, 4, 18, sd.data_ptr(), ld.data_ptr(), 1, 1, td.data_ptr(), 2, 0.1, 0,
                                qd.data_ptr(), 256, 64, None, None, None) == -1
    assert lib.qtz_kv_attention(None, cache._ref, qd.data_ptr(), 256, 64, 4, 18, sd.data_ptr(), ld.data_ptr(), 1, 1, td.data_ptr(), 2, 0.1, 0,
                                qd.data_ptr(), 256, 64, None, cache.workspace.data_ptr() if cache.workspace is not None else qd.data_ptr(), None) == -1
    assert lib.qtz_kv_attention_workspace_bytes(None, cache._ref) == 0
