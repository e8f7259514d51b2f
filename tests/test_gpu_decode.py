"""The serving calls together: steps of a quantized attention layer against float64 formulas of the same weights and cache."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_1806_08342_b200 import decode, qtz

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    return qtz.Handle(0)


def _real(h, w, group, dtype, symmetric):
    """The layer's weights in float64: the codes times their scales."""
    codes, scales, zeros = h.quantize_groups(w, group, dtype, symmetric)
    n, k = w.shape
    q = torch.stack((codes & 15, codes >> 4), -1).reshape(n, -1)[:, :k].double()
    at = torch.arange(k, device=w.device) // group
    if symmetric:
        q = torch.where(q > 7, q - 16, q)
    else:
        q = q - zeros[:, at].double()
    return q * scales[:, at].double()


@pytest.mark.parametrize("dtype,symmetric,window,q_heads,kv_heads", [(torch.bfloat16, True, 0, 8, 2), (torch.float16, False, 37, 3, 3)])
def test_steps_of_a_layer(handle, dtype, symmetric, window, q_heads, kv_heads):
    g = torch.Generator("cuda").manual_seed(7)
    hidden, dim, bt, group = 200, 64, 16, 64
    w_qkv = torch.randn((q_heads + 2 * kv_heads) * dim, hidden, device="cuda", generator=g) * hidden ** -0.5
    w_o = torch.randn(hidden, q_heads * dim, device="cuda", generator=g) * (q_heads * dim) ** -0.5
    layer = decode.AttentionLayer(handle, w_qkv, w_o, q_heads, kv_heads, dim, 40, bt, group, dtype, symmetric, window)
    rq, ro = _real(handle, w_qkv, group, dtype, symmetric), _real(handle, w_o, group, dtype, symmetric)
    requests = decode.Requests(handle, 4, 40, bt, 160)
    u = torch.finfo(dtype).eps / 2
    lens_want = [0] * 4
    for added in ([33, 1, 0, 70], [1, 1, 1, 1], [1, 0, 17, 5], [1, 1, 1, 1]):
        tokens = sum(added)
        x = torch.randn(tokens, hidden, device="cuda", generator=g).to(dtype)
        starts, lens, slots = requests.admit(torch.tensor(added, dtype=torch.int32, device="cuda"), tokens)
        y = layer(x, starts, lens, slots, requests.table)
        lens_want = [a + b for a, b in zip(lens_want, added)]
        assert not requests.refused and lens.tolist() == lens_want and requests.cached.tolist() == lens_want
        assert handle.device_status() == (0, 0)

        # q as the layer rounds it is within u |q| and the fp32 sum's error of the formula's q
        q = x.double() @ rq[:q_heads * dim].T
        slack = 2.0 ** -22 * hidden * (x.double().abs() @ rq[:q_heads * dim].abs().T)
        dq = (u * q.abs() + slack).view(tokens, q_heads, dim)
        q = q.view(tokens, q_heads, dim)
        attn, d_attn = torch.zeros_like(q), torch.zeros_like(q)
        row = 0
        for r, n in enumerate(added):
            pos = torch.arange(lens_want[r], device="cuda")
            at = requests.table[r, pos // bt].long() * bt + pos % bt
            k, v = (t.double() for t in layer.cache.read(at))          # code * scale: exact to 2^-24
            for i in range(n):
                p = lens_want[r] - n + i
                lo = max(0, p + 1 - window) if window else 0
                for hh in range(q_heads):
                    kk, vv = k[lo:p + 1, hh * kv_heads // q_heads], v[lo:p + 1, hh * kv_heads // q_heads]
                    logits = kk @ q[row, hh] * dim ** -0.5
                    # a logit moves by |dq| |k| and by the digits below 2^-22 of the largest q; a softmax by twice the largest move
                    move = ((kk.abs() @ (dq[row, hh] + 2.0 ** -20 * q[row, hh].abs().max())) * dim ** -0.5).max() + 2.0 ** -20 * (1 + logits.abs().max())
                    attn[row, hh] = torch.softmax(logits, 0) @ vv
                    d_attn[row, hh] = (torch.expm1(2 * move) + 2.0 ** -18) * vv.abs().max()
                row += 1
        attn, d_attn = attn.view(tokens, -1), d_attn.view(tokens, -1)
        d_attn = d_attn + u * (attn.abs() + d_attn)                     # y of the attention is rounded once
        want = attn @ ro.T
        bound = d_attn @ ro.abs().T
        bound = bound + 2.0 ** -22 * q_heads * dim * (attn.abs() @ ro.abs().T) + u * (want.abs() + bound) + torch.finfo(dtype).tiny
        worst = ((y.double() - want).abs() / bound).max().item()
        assert worst <= 1.0, worst


def test_release_and_refusal(handle):
    requests = decode.Requests(handle, 3, 6, 16, 64)
    add = lambda *n: torch.tensor(n, dtype=torch.int32, device="cuda")
    requests.admit(add(17, 16, 33), 66)
    assert not requests.refused and requests.free_count.item() == 0
    requests.admit(add(0, 1, 0), 1)                                     # no block left
    assert requests.refused and requests.cached.tolist() == [17, 16, 33] and requests.free_count.item() == 0
    mine = requests.table[2, :3].tolist()
    requests.release(2)
    assert requests.free_count.item() == 3 and sorted(requests.free[:3].tolist()) == sorted(mine)
    starts, lens, slots = requests.admit(add(0, 1, 20), 21)
    assert not requests.refused and lens.tolist() == [17, 17, 20] and requests.free_count.item() == 0
    used = [t for r, n in zip(requests.table.tolist(), (2, 2, 2)) for t in r[:n]]
    assert sorted(used) == list(range(6))


def test_command(handle, capsys):
    out = decode.main(["--requests", "3", "--prompt", "40", "--steps", "5", "--layers", "2", "--hidden", "256", "--q-heads", "4",
                       "--kv-heads", "2", "--head-dim", "64", "--block-tokens", "16"])
    # prompts 13, 26, 40; three steps before the capture, then five replays (the capture itself runs nothing)
    assert out["lens"] == [21, 34, 48] and "us a step" in capsys.readouterr().out
