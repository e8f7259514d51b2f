"""Softmax weights far below the largest one: a token that draws most of the weight and has no value to speak of, over a flat tail.

Bound of a row beside the output's rounding u, with c = softmax scale, p the exact probabilities, T the tiles of 128 tokens:
  logits   d_l = 2 (D + 8) 2^-24 c max_p sum |q k| + D 2^-24 c max|q| max|k|
  weights  relative: d_l twice, 2^-18 for exponentials, logarithms and scales, 4 T 2^-24 for the fp32 sums over the tiles
           absolute: half of 2^-31 of a tile's largest weight for each of its 128 tokens; the tiles' largest weights sum to
           1 at most, so that 2^-24 max|v| holds them twice over
  y        (2 d_l + 2^-18 + 4 T 2^-24) sum p |v| + 2^-24 max|v| + u |y| + 2^-25 of the type's subnormal step"""
import numpy as np
import pytest
import torch

from gpu_util import hq  # noqa: F401
from oracle import serving
from paper_1806_08342_b200 import qtz

pytestmark = pytest.mark.gpu

UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float16, torch.bfloat16)}


def strong_token(seed, lens, added, kv_heads, group, dim, block, dtype, gap, strong, k_scale=0.01, v_scale=0.02):
    """Logits of unit deviation but for token `strong` of each request, which lies `gap` above their mean and whose value is zero."""
    g = np.random.default_rng(seed)
    need = [-(-v // block) for v in lens]
    blocks = sum(need) + 2
    ids = g.permutation(blocks).astype(np.int32)
    table = np.zeros((len(lens), max(need)), np.int32)
    starts = np.concatenate(([0], np.cumsum(added))).astype(np.int32)
    base = g.normal(size=(kv_heads, 1, dim))
    # the rows of a head are nearly the same, so that one key is strong for all of them
    q = torch.from_numpy((base + 0.02 * g.normal(size=(int(starts[-1]), kv_heads, group, dim))).reshape(-1, kv_heads * group, dim)).to(dtype)
    size = np.sqrt((base ** 2).sum(-1))                                          # [kv_heads][1]
    codes = [np.clip(np.rint(g.normal(size=(blocks, kv_heads, block, dim)) * 12), -127, 127).astype(np.int8),
             g.integers(-127, 128, (blocks, kv_heads, block, dim)).astype(np.int8)]
    scale = float(1.0 / (12 * k_scale * size.mean()))
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
        for h in range(kv_heads):
            b, o = table[r, strong // block], strong % block
            codes[0][b, h, o] = np.clip(np.rint(base[h, 0] * gap / (scale * k_scale * size[h, 0] ** 2)), -127, 127)
            codes[1][b, h, o] = 0
    scales = [np.full((blocks, kv_heads), s, np.float32) for s in (k_scale, v_scale)]
    return codes, scales, table, starts, np.array(lens, np.int32), q, scale


def bound(q, codes, scales, starts, lens, table, scale, window, want, unit):
    q, dim, block = np.abs(q), q.shape[2], codes[0].shape[2]
    heads, kv_heads = q.shape[1], codes[0].shape[1]
    rel = np.zeros(q.shape[:2] + (1,))
    for r in range(len(lens)):
        used = table[r][:-(-int(lens[r]) // block)]
        for h in range(heads):
            g = h // (heads // kv_heads)
            k = (np.abs(codes[0][used, g].astype(np.float64)) * scales[0][used, g].astype(np.float64)[:, None, None]).reshape(-1, dim)
            for t in range(starts[r], starts[r + 1]):
                d = abs(scale) * (2 * (dim + 8) * 2.0 ** -24 * (k @ q[t, h]).max() + dim * 2.0 ** -24 * q[t, h].max() * k.max())
                rel[t, h] = 2 * d + 2.0 ** -18 + 4 * (lens[r] // 128 + 1) * 2.0 ** -24
    return rel, 2.0 ** -24 * max(127 * float(s.max()) for s in scales[1:])


def check(hq, made, window=0):
    codes, scales, table, starts, lens, q, scale = made
    cache = qtz.KvCache(hq, *(torch.from_numpy(c).cuda() for c in codes), *(torch.from_numpy(s).cuda() for s in scales))
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    y, lse = cache.attention(q.cuda(), dev(starts), dev(lens), dev(table), scale=scale, window=window, return_lse=True)
    qn = q.double().numpy()
    want, want_lse = serving.attention(qn, codes[0], scales[0], codes[1], scales[1], starts, lens, table, scale, window)
    size, _ = serving.attention(qn, codes[0], scales[0], np.abs(codes[1]), scales[1], starts, lens, table, scale, window)
    rel, absolute = bound(qn, codes, scales, starts, lens, table, scale, window, want, UNIT[q.dtype])
    tol = rel * size + absolute
    tol = tol + UNIT[q.dtype] * (np.abs(want) + tol) + (2.0 ** -25 if q.dtype is torch.float16 else 0)
    worst = (np.abs(y.double().cpu().numpy() - want) / tol).max()
    assert worst <= 1.0, worst
    assert np.abs(lse.double().cpu().numpy() - want_lse).max() <= rel.max() + 2.0 ** -18 * np.abs(want_lse).max()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("length,gap,strong", [(100, 15, 0), (700, 16, 0), (3000, 13, 1500), (13500, 16, 0), (40000, 17, 3)])
def test_one_request_cut_into_shares(hq, length, gap, strong, dtype):
    check(hq, strong_token(length + gap, [length], [1], 1, 4, 128, 32, dtype, gap, strong))


@pytest.mark.parametrize("dim,group,new", [(64, 1, 1), (64, 5, 1), (128, 4, 1), (128, 8, 1), (128, 4, 3), (128, 16, 1), (256, 2, 1), (256, 5, 2), (256, 16, 1)])
def test_items_within_one_share(hq, dim, group, new):
    """As many requests as leave most items whole, so that one part holds the strong token and the tail."""
    requests = 300 if dim < 256 else 160
    check(hq, strong_token(dim + group + new, [1100 + 3 * (i % 7) for i in range(requests)], [new] * requests, 1, group, dim, 64,
                           torch.float16, 16, 0))


def test_strong_token_last_and_in_a_window(hq):
    """The strong token comes after the tail, in the last tile and inside a window that leaves the first tiles out."""
    made = strong_token(5, [5000, 4100], [2, 2], 2, 4, 128, 16, torch.bfloat16, 15, 4097)
    check(hq, made)
    check(hq, made, window=3000)


@pytest.mark.parametrize("dtype,strong", [(torch.float16, 2.0 ** 15), (torch.bfloat16, 2.0 ** 20)])
@pytest.mark.parametrize("dim,group,new", [(64, 1, 1), (64, 5, 1), (128, 8, 1), (128, 5, 2), (128, 4, 3), (256, 16, 1)])
def test_strong_query_values_that_meet_codes_of_zero(hq, dim, group, new, dtype, strong):
    """One value of each query lies far above the others and meets nothing but zeros in the keys: the logits come from the others.
    A query loses half of 2^-29 of its largest value: a logit is off by c 2^-30 max|q| sum |k| beside the fp32 sums' part."""
    requests = 3
    codes, scales, table, starts, lens, q, scale = strong_token(dim + group, [260, 131, 70], [new] * requests, 2, group, dim, 16, dtype, 2, 0)
    at = 7
    codes[0][..., at] = 0
    q[:, :, at] = strong
    cache = qtz.KvCache(hq, *(torch.from_numpy(c).cuda() for c in codes), *(torch.from_numpy(s).cuda() for s in scales))
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    y, lse = cache.attention(q.cuda(), dev(starts), dev(lens), dev(table), scale=scale, return_lse=True)
    qn = q.double().numpy()
    args = (scales[1], starts, lens, table, scale)
    want, want_lse = serving.attention(qn, codes[0], scales[0], codes[1], *args)
    size, _ = serving.attention(qn, codes[0], scales[0], np.abs(codes[1]), *args)
    rest = qn.copy()
    rest[..., at] = 0
    k = np.abs(codes[0].astype(np.float64)).sum(-1).max() * scales[0].max()                # sum |k| of a token, at most
    d = scale * (2 * (dim + 8) * 2.0 ** -24 * np.abs(rest).max() * k + 2.0 ** -30 * strong * k)
    tol = (2 * d + 2.0 ** -18) * size + 2.0 ** -24 * 127 * scales[1].max()
    tol = tol + UNIT[dtype] * (np.abs(want) + tol) + 2.0 ** -25
    assert (np.abs(y.double().cpu().numpy() - want) <= tol).all()
    assert np.abs(lse.double().cpu().numpy() - want_lse).max() <= d + 2.0 ** -18 * (1 + np.abs(want_lse).max())
