"""Decoding with quantized attention layers: 4-bit weights, a paged 8-bit key/value cache.

The serving calls of the library run together as a server would use them: `Requests` admits the tokens of a step and
hands out cache blocks on the device (`qtz_kv_schedule`); an `AttentionLayer` projects them (`qtz_linear_w4`), quantizes
the new keys and values into its cache (`qtz_kv_append`), attends (`qtz_kv_attention`) and projects back.  Nothing is
copied to the host between the steps, so that a step can be captured in a CUDA graph and replayed.

    python -m paper_1806_08342_b200.decode --requests 16 --prompt 500 --steps 64

admits prompts of ragged lengths, then decodes one token a request and step, with seeded random weights and activations.  With
`--ffn 5504` each layer is a whole block: norms of the residual stream (`qtz_f8_rmsnorm`) before the attention and before a gated
feed-forward part whose products run in 8-bit floating point (`qtz_f8_quantize`, `qtz_f8_linear`).
"""
from __future__ import annotations

import argparse

import torch

from . import qtz


class Requests:
    """Lengths, block tables and free blocks of up to `count` requests that are served together."""

    def __init__(self, handle: qtz.Handle, count: int, blocks: int, block_tokens: int, most_tokens: int):
        device = f"cuda:{handle.device}"
        self.h, self.block_tokens = handle, block_tokens
        self.cached = torch.zeros(count, dtype=torch.int32, device=device)
        self.table = torch.full((count, -(-most_tokens // block_tokens)), -1, dtype=torch.int32, device=device)
        self.free = torch.arange(blocks, dtype=torch.int32, device=device)
        self.free_count = torch.full((1,), blocks, dtype=torch.int32, device=device)
        self.report = None

    def admit(self, added, capacity: int):
        """added [count] int32 on the device, `capacity` tokens at most: (starts, lens, slots) of the step.  If the blocks do
        not suffice nothing is admitted and `refused` says so."""
        starts, lens, slots, self.report = self.h.kv_schedule(self.cached, added, self.table, self.free, self.free_count,
                                                              self.block_tokens, capacity)
        self.cached.copy_(lens)
        self.free_count.copy_(self.report[:1])
        return starts, lens, slots

    @property
    def refused(self) -> bool:
        """Whether the last step was refused (reads one value from the device)."""
        return self.report is not None and bool(self.report[3].item())

    def release(self, request: int) -> None:
        """Ends a request: its blocks are free again (reads two values from the device)."""
        used = -(-int(self.cached[request].item()) // self.block_tokens)
        have = int(self.free_count.item())
        self.free[have:have + used] = self.table[request, :used]
        self.table[request].fill_(-1)
        self.free_count += used
        self.cached[request] = 0


class AttentionLayer:
    """y = W_o attention(W_q x, W_k x, W_v x) with the weights in 4 bits and the keys and values of all tokens so far in 8."""

    def __init__(self, handle: qtz.Handle, w_qkv, w_o, q_heads: int, kv_heads: int, head_dim: int, blocks: int,
                 block_tokens: int, group: int = 128, dtype=torch.bfloat16, symmetric: bool = True, window: int = 0):
        """w_qkv [(q_heads + 2 kv_heads) head_dim][hidden] and w_o [hidden][q_heads head_dim] in fp32 on the device."""
        self.q_heads, self.kv_heads, self.head_dim, self.window = q_heads, kv_heads, head_dim, window
        self.qkv, self.out = (self._linear(handle, w, group, dtype, symmetric) for w in (w_qkv, w_o))
        self.cache = handle.kv_cache(blocks, kv_heads, block_tokens, head_dim)

    @staticmethod
    def _linear(handle, w, group, dtype, symmetric):
        codes, scales, zeros = handle.quantize_groups(w, group, dtype, symmetric)
        return handle.linear_create(codes, scales, w.shape[1], group, zeros)

    def __call__(self, x, starts, lens, slots, table):
        """x [tokens][hidden] of the step that `Requests.admit` described."""
        qkv = self.qkv(x).view(x.shape[0], self.q_heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = qkv.split_with_sizes((self.q_heads, self.kv_heads, self.kv_heads), dim=1)
        self.cache.append(k, v, slots)
        y = self.cache.attention(q, starts, lens, table, window=self.window)
        return self.out(y.view(x.shape[0], -1))


class FeedForward:
    """x' = W_down (silu(W_gate n) * W_up n), n = norm(x + residual) * gain, with e4m3 weights and activations."""

    def __init__(self, handle: qtz.Handle, gain, w_gate_up, w_down, eps: float = 1e-6):
        """w_gate_up [2 width][hidden], the gate's rows first, and w_down [hidden][width] in any of the three types on the device; width a
        multiple of 8; gain [hidden] in the layer's type."""
        self.handle, self.gain, self.eps, self.width = handle, gain, eps, w_down.shape[1]
        if w_gate_up.shape != (2 * self.width, w_down.shape[0]) or self.width % 8:
            raise ValueError("expected weights [2 width][hidden] and [hidden][width], width a multiple of 8")
        self.gate_up, self.down = (handle.f8_linear_create(*handle.f8_quantize_weights(w)) for w in (w_gate_up, w_down))

    def __call__(self, x, residual=None):
        """(x', x + residual) of x [tokens][hidden]; without a residual the second is x."""
        codes, scales, _, total = self.handle.f8_rmsnorm(x, self.gain, self.eps, residual=residual)
        both = self.gate_up(codes, scales, dtype=x.dtype)
        codes, scales = self.handle.f8_quantize(both[:, self.width:], gate=both[:, :self.width])
        return self.down(codes, scales, dtype=x.dtype), x if residual is None else total


class Block:
    """An attention layer and a feed-forward part, each behind a norm of the residual stream."""

    def __init__(self, attention: AttentionLayer, gain, feed_forward: FeedForward):
        self.attention, self.gain, self.feed_forward = attention, gain, feed_forward

    def __call__(self, x, residual, starts, lens, slots, table):
        """(x', residual') of x [tokens][hidden] and the residual stream, None before the first block."""
        ff = self.feed_forward
        _, _, values, total = ff.handle.f8_rmsnorm(x, self.gain, ff.eps, residual=residual, codes=False, values=True)
        return ff(self.attention(values, starts, lens, slots, table), x if residual is None else total)


def run_blocks(blocks, x, starts, lens, slots, table):
    """Hidden states behind `blocks` of x [tokens][hidden]: the residual stream with what the last block adds to it."""
    residual = None
    for block in blocks:
        x, residual = block(x, residual, starts, lens, slots, table)
    return x if residual is None else x + residual


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("requests", 16), ("prompt", 500), ("steps", 64), ("layers", 4), ("hidden", 2048), ("q-heads", 16),
                        ("kv-heads", 4), ("head-dim", 128), ("block-tokens", 32), ("group", 128), ("window", 0), ("seed", 0), ("ffn", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    o = ap.parse_args(argv)
    h = qtz.Handle(0)
    g = torch.Generator("cuda").manual_seed(o.seed)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    warm = 3
    most = o.prompt + o.steps + warm
    blocks = o.requests * -(-most // o.block_tokens)
    requests = Requests(h, o.requests, blocks, o.block_tokens, most)
    width = (o.q_heads + 2 * o.kv_heads) * o.head_dim
    layers = [AttentionLayer(h, randn(width, o.hidden) * o.hidden ** -0.5, randn(o.hidden, o.q_heads * o.head_dim) * (o.q_heads * o.head_dim) ** -0.5,
                             o.q_heads, o.kv_heads, o.head_dim, blocks, o.block_tokens, o.group, window=o.window)
              for _ in range(o.layers)]
    if o.ffn:
        layers = [Block(layer, randn(o.hidden).bfloat16(), FeedForward(h, randn(o.hidden).bfloat16(), randn(2 * o.ffn, o.hidden) * o.hidden ** -0.5,
                                                                       randn(o.hidden, o.ffn) * o.ffn ** -0.5)) for layer in layers]

    def step(x, added):
        plan = requests.admit(added, x.shape[0])
        if o.ffn:
            return run_blocks(layers, x, *plan, requests.table)
        for layer in layers:
            x = layer(x, *plan, requests.table)
        return x

    lengths = [max(1, o.prompt * (r + 1) // o.requests) for r in range(o.requests)]      # ragged prompts
    step(randn(sum(lengths), o.hidden).bfloat16(), torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    if requests.refused:
        raise RuntimeError("the prompts do not fit into the cache")
    one, x = torch.ones(o.requests, dtype=torch.int32, device="cuda"), randn(o.requests, o.hidden).bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(warm):
            step(x, one)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step(x, one)
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(o.steps):
        graph.replay()
    stop.record()
    torch.cuda.synchronize()
    if requests.refused or not bool(torch.isfinite(y).all()):
        raise RuntimeError("the steps were refused or gave no numbers")
    rc, site = h.device_status()
    if rc:
        raise RuntimeError(f"device status {rc} at {site}")
    us = start.elapsed_time(stop) * 1e3 / o.steps
    print(f"{o.layers} {'blocks' if o.ffn else 'attention layers'}, {o.requests} requests, {sum(lengths)} prompt tokens: {us:.1f} us a step, "
          f"{o.requests / us * 1e6:.0f} tokens/s")
    return {"us_per_step": us, "lens": requests.cached.tolist()}


if __name__ == "__main__":
    main()
