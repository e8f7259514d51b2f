"""The widest layer and the longest request that the serving calls are measured with, against float64 on the GPU.

Bounds: the linear layers' is that of fp32 sums in any order, 2 (k + 8) 2^-24 sum |x w|, and half of 2^-29 of a block's largest value for
each of its 256 columns; the attention's that of one strong token's tests: relative 2 d_l + 2^-18 + 4 T 2^-24 with d_l the logits' error
and T the tiles of 128 tokens, 2^-24 max|v| beside it.  Both add half a unit of the output's type."""
import math

import pytest
import torch

from gpu_util import hq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("zeros,group,dtype", [(False, 128, torch.bfloat16), (True, 64, torch.float16)])
def test_widest_layer(hq, zeros, group, dtype):
    n, k = 28672, 8192
    g = torch.Generator("cuda").manual_seed(group)
    codes = torch.randint(0, 256, (n, k // 2), device="cuda", dtype=torch.uint8, generator=g)
    scales = (torch.rand(n, k // group, device="cuda", generator=g) * 0.01 + 0.001).to(dtype)
    z = torch.randint(0, 16, (n, k // group), device="cuda", dtype=torch.uint8, generator=g) if zeros else None
    plan = hq.linear_create(codes, scales, k, group, zeros=z)
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(1).double().view(n, k // group, group)
    w = ((q - z.double()[..., None] if zeros else torch.where(q > 7, q - 16, q)) * scales.double()[..., None]).view(n, k)
    del q
    for rows in (1, 3, 8, 32, 70):
        x = torch.randn(rows, k, device="cuda", generator=g)
        x[:, ::199] *= 30.0
        x = x.to(dtype)
        got, want = plan(x).double(), x.double() @ w.T
        tol = 2 * (k + 8) * 2.0 ** -24 * (x.double().abs() @ w.abs().T)
        for b in range(0, k, 256):
            tol += 2.0 ** -29 * x[:, b:b + 256].double().abs().amax(1, keepdim=True) * w[:, b:b + 256].abs().sum(1)
        tol = tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol) + 2.0 ** -25
        assert ((got - want).abs() / tol).max().item() <= 1.0


@pytest.mark.parametrize("dim,group,added,block,window", [(128, 8, 1, 64, 0), (128, 4, 1, 32, 0), (64, 3, 4, 16, 0), (256, 2, 2, 128, 0), (128, 5, 3, 16, 100_000)])
def test_longest_request(hq, dim, group, added, block, window):
    length, heads, dtype = 262_143, 2, torch.bfloat16
    g = torch.Generator("cuda").manual_seed(dim + group)
    blocks = -(-length // block)
    cache = hq.kv_cache(blocks, heads, block, dim)
    for t in (cache.k, cache.v):
        t.random_(-127, 128, generator=g)
    for t in (cache.k_scale, cache.v_scale):
        t.uniform_(0.005, 0.03, generator=g)
    table = torch.randperm(blocks, device="cuda", generator=g).int()[None]
    q = (torch.randn(added, heads * group, dim, device="cuda", generator=g) * 0.7).to(dtype)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    y, lse = cache.attention(q, ints(0, added), ints(length), table, window=window, return_lse=True)
    ids, c = table[0].long(), dim ** -0.5
    for h in range(heads):
        k, v = ((t[ids, h].double() * s[ids, h].double()[:, None, None]).flatten(0, 1)[:length] for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        for i in range(added):
            end = length - added + i + 1
            begin = max(0, end - window) if window else 0
            kk, vv, qq = k[begin:end], v[begin:end], q[i, h * group:(h + 1) * group].double()
            t = qq @ kk.T * c
            p = torch.softmax(t, -1)
            want, size = p @ vv, p @ vv.abs()
            d = c * (2 * (dim + 8) * 2.0 ** -24 * (qq.abs() @ kk.abs().T).amax(1) + dim * 2.0 ** -30 * qq.abs().amax(1) * kk.abs().max())[:, None]
            tol = (2 * d + 2.0 ** -18 + 4 * (length // 128 + 1) * 2.0 ** -24) * size + 2.0 ** -24 * 127 * cache.v_scale.max().double()
            tol = tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol)
            got = y[i, h * group:(h + 1) * group].double()
            assert ((got - want).abs() / tol).max().item() <= 1.0
            top = torch.logsumexp(t, -1)
            off = (lse[i, h * group:(h + 1) * group].double() - top).abs()
            assert (off <= d[:, 0] + 4 * (length // 128 + 1) * 2.0 ** -24 + 2.0 ** -18 * (1 + top.abs())).all()
    assert math.isfinite(float(y.float().sum()))
