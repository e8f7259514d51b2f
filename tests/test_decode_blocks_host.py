"""Blocks of the decoding example against the formula h = h + attention(norm(h)), h = h + feed_forward(norm(h)), on the CPU: the calls of
the library are replaced by their formulas in 64 bits."""
import pytest
import torch

from paper_1806_08342_b200 import decode


class Formulas:
    """The calls of `qtz.Handle` that the blocks make, without quantization."""

    @staticmethod
    def f8_rmsnorm(x, gain, eps=1e-6, residual=None, codes=True, values=False):
        h = x if residual is None else x + residual
        v = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * gain
        return v if codes else None, None, v if values else None, None if residual is None else h

    @staticmethod
    def f8_quantize(x, gate=None):
        return (x if gate is None else x * gate / (1 + torch.exp(-gate))), None

    @staticmethod
    def f8_quantize_weights(w):
        return w, None

    @staticmethod
    def f8_linear_create(w, scales):
        return lambda x, scales, dtype: x @ w.T


@pytest.mark.parametrize("count", [1, 2, 5])
def test_blocks_are_the_formula(count):
    g = torch.Generator().manual_seed(count)
    rand = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    tokens, hidden, width = 7, 24, 40
    x, want, blocks = rand(tokens, hidden), None, []
    for _ in range(count):
        mix, gains, wide, down = rand(tokens, tokens), rand(2, hidden), rand(2 * width, hidden) / 5, rand(hidden, width) / 6
        attention = lambda v, starts, lens, slots, table, mix=mix: mix @ v + table  # noqa: E731
        blocks.append(decode.Block(attention, gains[0], decode.FeedForward(Formulas(), gains[1], wide, down, 1e-5)))
        norm = lambda h, gain: h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5) * gain  # noqa: E731
        want = x if want is None else want
        want = want + mix @ norm(want, gains[0]) + 3
        both = norm(want, gains[1]) @ wide.T
        want = want + (both[:, width:] * torch.nn.functional.silu(both[:, :width])) @ down.T
    got = decode.run_blocks(blocks, x, None, None, None, 3)
    # five blocks of a few dozen operations, each off by 2^-53 of values that grow to a few hundred at most
    assert (got - want).abs().max() <= 2.0 ** -40 * want.abs().max()


def test_no_blocks_change_nothing():
    x = torch.ones(2, 3)
    assert decode.run_blocks([], x, None, None, None, None) is x
