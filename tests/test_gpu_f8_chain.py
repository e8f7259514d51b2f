"""The 8-bit floating-point calls as they are used together: a gated feed-forward part and whole blocks of the decoding example."""
import numpy as np
import pytest
import torch

from oracle import f8
from paper_1806_08342_b200 import decode, qtz

pytestmark = pytest.mark.gpu

UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float16, torch.bfloat16, torch.float32)}


@pytest.fixture(scope="module")
def handle():
    h = qtz.Handle(0)
    yield h
    assert h.device_status() == (0, 0)


def f64(t):
    return t.double().cpu().numpy()


def real(codes, scales):
    """Values of codes with a scale for each row and 128 columns."""
    c = f8.decode(codes.contiguous().view(torch.uint8).cpu().numpy())
    return c * f8.spread(f64(scales), *c.shape)


def check_product(y, codes, scales, w):
    """Against the formula on the codes at hand: 2 (k + 8) 2^-24 of the products' magnitudes, and half a unit of y."""
    wc, ws = w
    want, size = f8.linear(codes.contiguous().view(torch.uint8).cpu().numpy(), f64(scales), wc.view(torch.uint8).cpu().numpy(), f64(ws))
    tol = 2 * (wc.shape[1] + 8) * 2.0 ** -24 * size
    assert (np.abs(f64(y) - want) <= tol + UNIT[y.dtype] * (np.abs(want) + tol) + 2.0 ** -25).all()


def check_codes(codes, scales, v, off):
    """Half a step of e4m3, what the value is off by, and the fp32 steps of scale and quotient."""
    s = f8.spread(f64(scales), *v.shape)
    assert (np.abs(real(codes, scales) - v) <= f8.half_step(np.minimum(np.abs(v) / s, 447.0)) * s + np.abs(v) * (off + 2.0 ** -21)).all()


@pytest.mark.parametrize("tokens", [1, 7, 40, 130, 700])
@pytest.mark.parametrize("dtype", list(UNIT))
def test_feed_forward(handle, tokens, dtype):
    g = torch.Generator("cuda").manual_seed(tokens)
    hidden, width = 328, 1000
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, residual, gain = rand(tokens, hidden).to(dtype), (3 * rand(tokens, hidden)).to(dtype), (1 + 0.2 * rand(hidden)).to(dtype)
    wide, down = rand(2 * width, hidden) * hidden ** -0.5, rand(hidden, width) * width ** -0.5
    layer = decode.FeedForward(handle, gain, wide, down, 1e-5)
    for res in (residual, None):
        y, total = layer(x, res)
        codes, scales, _, same = handle.f8_rmsnorm(x, gain, 1e-5, residual=res)
        h, n = f8.rmsnorm(f64(x), f64(gain), 1e-5, None if res is None else f64(res))
        check_codes(codes, scales, n, 2.0 ** -18)
        if res is None:
            assert total is x
        else:
            assert torch.equal(total, same) and (np.abs(f64(total) - h) <= np.abs(h) * (UNIT[dtype] + 2.0 ** -23)).all()
        both = layer.gate_up(codes, scales, dtype=dtype)
        check_product(both, codes, scales, handle.f8_quantize_weights(wide))
        codes, scales = handle.f8_quantize(both[:, width:], gate=both[:, :width])
        check_codes(codes, scales, f8.gated(f64(both[:, width:]), f64(both[:, :width])), 2.0 ** -16)
        check_product(y, codes, scales, handle.f8_quantize_weights(down))
        assert torch.equal(layer.down(codes, scales, dtype=dtype), y)


def test_captured_replayed_and_on_another_stream(handle):
    """A graph of the layer, replayed on new inputs, beside eager calls and a second graph of another size."""
    g = torch.Generator("cuda").manual_seed(1)
    hidden, width = 512, 768
    layer = decode.FeedForward(handle, torch.ones(hidden, device="cuda", dtype=torch.bfloat16), torch.randn(2 * width, hidden, device="cuda", generator=g) * 0.05,
                               torch.randn(hidden, width, device="cuda", generator=g) * 0.05)
    side = torch.cuda.Stream()
    graphs = []
    for tokens in (3, 300):
        x, residual = (torch.randn(tokens, hidden, device="cuda", generator=g).bfloat16() for _ in range(2))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            layer(x, residual)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = layer(x, residual)
        graphs.append((graph, x, residual, out))
    for _ in range(3):
        for graph, x, residual, out in graphs:
            x.normal_(generator=g)
            residual.normal_(generator=g)
            want = [t.clone() for t in layer(x, residual)]
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                again = layer(x, residual)
            torch.cuda.current_stream().wait_stream(side)
            assert all(torch.equal(a, b) for a, b in zip(again, want))


def test_rows_of_a_batch_do_not_depend_on_each_other(handle):
    """Padding a batch, with NaN even, changes nothing in its other rows, as long as the number of rows takes the same way."""
    g = torch.Generator("cuda").manual_seed(2)
    n, k = 700, 900
    w = torch.randn(n, k, device="cuda", generator=g) * 0.03
    plan = handle.f8_linear_create(*handle.f8_quantize_weights(w))
    x = torch.randn(64, 904, device="cuda", generator=g).bfloat16()[:, :k]
    codes, scales = handle.f8_quantize(x)
    want = plan(codes, scales)
    x[40:] = float("nan")
    padded, padded_scales = handle.f8_quantize(x)
    got = plan(padded, padded_scales)
    assert torch.equal(got[:40], want[:40]) and bool(got[40:].isnan().all())


@pytest.mark.parametrize("rows", [2, 90, 400])
def test_a_layer_on_two_streams_at_once(handle, rows):
    g = torch.Generator("cuda").manual_seed(rows)
    plan = handle.f8_linear_create(*handle.f8_quantize_weights(torch.randn(2000, 1500, device="cuda", generator=g)))
    inputs = [handle.f8_quantize(torch.randn(rows, 1500, device="cuda", generator=g)[:, :1500]) for _ in range(2)]
    want = [plan(*i) for i in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in inputs]
    got = [[], []]
    for _ in range(20):
        for i, (stream, one) in enumerate(zip(streams, inputs)):
            with torch.cuda.stream(stream):
                got[i].append(plan(*one))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in range(2) for y in got[i])


def test_blocks_of_the_example():
    got = decode.main(["--requests", "4", "--prompt", "150", "--steps", "4", "--layers", "2", "--hidden", "512", "--q-heads", "8", "--kv-heads", "2",
                       "--head-dim", "64", "--ffn", "1376"])
    assert got["lens"] == [max(1, 150 * (r + 1) // 4) + 3 + 4 for r in range(4)] and got["us_per_step"] > 0


def test_feed_forward_refuses_weights_that_do_not_chain(handle):
    gain = torch.ones(64, device="cuda")
    for wide, down in (((200, 64), (64, 96)), ((192, 64), (60, 96)), ((200, 64), (64, 100))):
        with pytest.raises(ValueError):
            decode.FeedForward(handle, gain, torch.zeros(*wide, device="cuda"), torch.zeros(*down, device="cuda"))


LEAST, USUAL = 1000, 2_000_000_000


@pytest.mark.parametrize("case", [(1, 4096, 8192), (30, 5000, 2048), (128, 1000, 1024), (200, 2000, 8192), (1000, 4096, 1024)])
def test_products_under_the_least_wait_budget_and_the_ones_after_them(case):
    """A wait that runs out ends the call by itself and is reported; the next calls are right either way."""
    rows, n, k = case
    h = qtz.Handle(0)
    g = torch.Generator("cuda").manual_seed(3)
    plan = h.f8_linear_create(*h.f8_quantize_weights(torch.randn(n, k, device="cuda", generator=g)))
    codes, scales = h.f8_quantize(torch.randn(rows, k, device="cuda", generator=g))
    want = plan(codes, scales)
    assert h.device_status() == (0, 0)
    cold = torch.empty(64 << 20, device="cuda")                          # more than the caches hold
    for _ in range(4):
        cold.fill_(1)
        h.set_wait_budget(LEAST)
        got = plan(codes, scales)
        torch.cuda.synchronize()
        status = h.device_status()
        assert status == (-7, 14) or (status == (0, 0) and torch.equal(got, want))
        h.set_wait_budget(USUAL)
        for _ in range(2):
            assert torch.equal(plan(codes, scales), want)
        assert h.device_status() == (0, 0)
    plan.close()
    h.close()
