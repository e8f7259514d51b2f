"""Definitions of the serving operators in fp64 numpy -- TEST INFRASTRUCTURE.

4-bit linear layers (Sections 2.1, 2.2 with one scale per group of columns), admission of a decoding step, the 8-bit
key/value cache and attention over it.  Written from the formulas with loops over requests, blocks and heads; shares
nothing with the CUDA library.
"""
from __future__ import annotations

import numpy as np

MIN_SCALE = 2.0 ** -100


def unpack4(packed, k, signed):
    """[n][(k + 1) // 2] bytes -> [n][k] codes: element 2i in the low nibble, 2i + 1 in the high one."""
    out = np.zeros((packed.shape[0], 2 * packed.shape[1]), np.int64)
    out[:, 0::2] = packed % 16
    out[:, 1::2] = packed // 16
    out = out[:, :k]
    return np.where(out >= 8, out - 16, out) if signed else out


def linear(x, codes, scales, zeros, bias, k, group, signed):
    q = unpack4(codes, k, signed).astype(np.float64)
    g = np.arange(k) // group
    if zeros is not None:
        q -= np.minimum(zeros, 15).astype(np.float64)[:, g]
    y = x.astype(np.float64) @ (q * scales.astype(np.float64)[:, g]).T
    return y if bias is None else y + bias.astype(np.float64)


def schedule(cached, added, table, free, block, capacity):
    """(table, starts, lens, slots, report); all or nothing."""
    cached, added, table = [int(c) for c in cached], [int(m) for m in added], np.array(table)
    blocks_of = lambda v: -(-v // block)  # noqa: E731
    refused = min(cached + added) < 0 or sum(added) > capacity
    refused = refused or any(blocks_of(c + m) > table.shape[1] for c, m in zip(cached, added))
    refused = refused or sum(blocks_of(c + m) - blocks_of(c) for c, m in zip(cached, added)) > len(free)
    starts, lens, slots, left = [0], [], [], len(free)
    for r, (c, m) in enumerate(zip(cached, added)):
        if refused:
            starts.append(0)
            lens.append(c)
            continue
        for j in range(blocks_of(c), blocks_of(c + m)):
            left -= 1
            table[r, j] = free[left]
        slots += [int(table[r, p // block]) * block + p % block for p in range(c, c + m)]
        starts.append(len(slots))
        lens.append(c + m)
    report = [left, len(slots), len(free) - left, int(refused)]
    slots += [-1] * (capacity - len(slots))
    return table, np.array(starts, np.int32), np.array(lens, np.int32), np.array(slots, np.int64), np.array(report, np.int32)


def append(codes, scale, x, slots):
    """One tensor of the cache after an append, in the fp32 steps of the definition (bit for bit): codes
    [blocks][heads][block][dim], scale [blocks][heads], x [tokens][heads][dim]."""
    codes, scale, x = codes.copy(), scale.astype(np.float32).copy(), x.astype(np.float32)
    f = np.float32
    block = codes.shape[2]
    runs = {}
    for i, s in enumerate(slots):
        if s >= 0:
            runs.setdefault(int(s) // block, []).append((int(s) % block, i))
    for b, run in runs.items():
        offsets, rows = [o for o, _ in run], [i for _, i in run]
        for h in range(codes.shape[1]):
            v = x[rows, h]
            finite = np.abs(v[np.isfinite(v)])
            s = max(f(finite.max() if finite.size else 0.0) / f(127.0), f(MIN_SCALE))
            if offsets[0] > 0:
                old = max(scale[b, h], f(MIN_SCALE))
                if old < s:
                    codes[b, h, :offsets[0]] = np.rint(codes[b, h, :offsets[0]].astype(f) * (old / s)).astype(np.int8)
                s = max(s, old)
            scale[b, h] = s
            with np.errstate(invalid="ignore", over="ignore"):
                q = np.rint(v / s)
            q = np.where(np.isnan(q), -127.0, np.clip(q, -127.0, 127.0))
            codes[b, h, offsets] = q.astype(np.int8)
    return codes, scale


def read(codes, scale, slots):
    """fp32 values [tokens][heads][dim]: one fp32 product each."""
    block = codes.shape[2]
    out = np.zeros((len(slots), codes.shape[1], codes.shape[3]), np.float32)
    for i, s in enumerate(slots):
        if s >= 0:
            b, o = int(s) // block, int(s) % block
            out[i] = codes[b, :, o].astype(np.float32) * np.maximum(scale[b], np.float32(MIN_SCALE))[:, None]
    return out


def attention(q, codes_k, scale_k, codes_v, scale_v, starts, lens, table, scale, window=0):
    """(y, lse) in fp64; rows that see nothing give zeros and -inf."""
    q = q.astype(np.float64)
    tokens, heads, dim = q.shape
    kv_heads, block = codes_k.shape[1], codes_k.shape[2]
    y, lse = np.zeros((tokens, heads, dim)), np.full((tokens, heads), -np.inf)
    for r in range(len(lens)):
        length, ids = int(lens[r]), table[r]
        used = ids[:-(-length // block)] if length > 0 else ids[:0]
        for g in range(kv_heads):
            real = lambda c, s: (c[used, g].astype(np.float64) * np.maximum(s[used, g], MIN_SCALE).astype(np.float64)[:, None, None]).reshape(-1, dim)  # noqa: E731
            k, v = real(codes_k, scale_k), real(codes_v, scale_v)
            for t in range(int(starts[r]), int(starts[r + 1])):
                end = length - (int(starts[r + 1]) - t) + 1
                begin = max(0, end - window) if window else 0
                if end <= begin:
                    continue
                for h in range(g * (heads // kv_heads), (g + 1) * (heads // kv_heads)):
                    s = k[begin:end] @ q[t, h] * scale
                    top = s.max()
                    p = np.exp(s - top)
                    y[t, h] = p @ v[begin:end] / p.sum()
                    lse[t, h] = top + np.log(p.sum())
    return y, lse
