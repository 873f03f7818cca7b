"""The operators for long contexts on the 8-bit KV cache in 64 bits on the CPU: their definitions, written as loops, and error bounds."""
import numpy as np
import torch

import _kv8 as K


def rotate(x, positions, freq, pairs):
    """x: float64 [rows, heads, dim], freq: fp32 [pairs].  Rotated in 64 bits by cosines and sines rounded to fp32, and how large the
    two terms of each element are together."""
    half = freq.shape[0]
    angle = np.asarray(positions, dtype=np.float64)[:, None] * freq.astype(np.float64)
    c, s = (f(angle).astype(np.float32).astype(np.float64)[:, None] for f in (np.cos, np.sin))
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    y, size = x.copy(), np.abs(x)
    with np.errstate(invalid="ignore"):
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., i] * s + x[..., j] * c
        size[..., i] = size[..., j] = np.maximum(np.abs(x[..., i] * c) + np.abs(x[..., j] * s), np.abs(x[..., i] * s) + np.abs(x[..., j] * c))
    return y, size


STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def rotated_error(y, size, dtype):
    """fp32 comes out of 64 bits rounded once.  16 bits: two products and a sum in fp32 (three roundings, of terms no larger than size), one
    more to the type; fp16 holds nothing below 2^-25."""
    e = STEP[dtype] * np.abs(y)
    if dtype != torch.float32:
        e = e * (1 + 2.0 ** -10) + 3 * K.F * size * (1 + STEP[dtype])
    return e + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -140)


def places(spans, total):
    """The place of every new token in its request, None for rows that no request has."""
    at = [None] * total
    for _, start, new, length in spans:
        for i in range(new):
            at[start + i] = length - new + i
    return at


def bound(cache, spans, bounds):
    """bounds: uint8 [blocks, heads, 2, dim], changed in place."""
    for row, _, new, length in spans:
        for block in range(max(length - new, 0) // cache.bs, -(-length // cache.bs) if new and length > 0 else 0):
            e = cache.entry(row, block)
            if e < 0:
                continue
            codes = cache.code[0][e, :min(cache.bs, length - block * cache.bs)]
            x = K.CODES[codes]
            with np.errstate(invalid="ignore"):
                for k, pick in enumerate((x.min(0), x.max(0))):
                    bounds[e, :, k] = np.where(np.isnan(pick), 127, K.nearest_code(np.nan_to_num(pick)))


def select(cache, spans, bounds, q, group, n_select, first, recent, blocks):
    """blocks: int32 [total, heads, n_select], changed in place."""
    b = K.CODES[bounds]
    for row, start, new, length in spans:
        for i in range(new):
            p = length - new + i
            seen = p // cache.bs + 1 if p >= 0 else 0
            for h in range(cache.heads):
                if seen <= n_select:
                    taken = list(range(seen))
                else:
                    score = []
                    for j in range(first, seen - recent):
                        e = cache.entry(row, j)
                        s = -np.inf
                        if e >= 0:
                            with np.errstate(invalid="ignore"):
                                each = [np.maximum(q[start + i, g] * b[e, h, 0], q[start + i, g] * b[e, h, 1]).sum() for g in range(h * group, (h + 1) * group)]
                            s = max(each) * cache.scale[0][e, h] if not np.isnan(each).any() else -np.inf
                        score.append((-s, j))
                    taken = list(range(first)) + sorted(j for _, j in sorted(score)[:n_select - first - recent]) + list(range(seen - recent, seen))
                blocks[start + i, h] = taken + [-1] * (n_select - len(taken))


class _Listed:
    """One head's listed tokens as a context of their own."""

    def __init__(self, k, v, there):
        self.heads, self.kv, self.there = 1, (k, v), there

    def tokens(self, kv, row, length):
        return self.kv[kv], self.there


def attend_blocks(cache, spans, blocks, q, scale, group, dtype):
    """out, lse, and for each the largest error allowed: those of _kv8.attend, over the listed tokens."""
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    d_out, d_lse = np.zeros(q.shape), np.zeros(q.shape[:2])
    for row, start, new, length in spans:
        whole = [cache.tokens(kv, row, length) for kv in (0, 1)] if length > 0 else None
        for i in range(start, start + new):
            seen = length - new + i - start + 1
            if seen <= 0:
                continue
            count = min(blocks.shape[2], (seen - 1) // cache.bs + 1)
            for h in range(cache.heads):
                at = [int(j) * cache.bs + s for j in blocks[i, h, :count] if 0 <= j <= (seen - 1) // cache.bs for s in range(cache.bs)]
                at = np.array([t for t in at if t < seen], dtype=np.int64)
                if not len(at):
                    continue
                g = slice(h * group, (h + 1) * group)
                one = _Listed(whole[0][0][at][:, h:h + 1], whole[1][0][at][:, h:h + 1], whole[0][1][at])
                (o, l, _), (do, dl, _) = K.attend(one, [(0, 0, 1, len(at))], q[i:i + 1, g], scale, group, dtype)
                out[i, g], lse[i, g], d_out[i, g], d_lse[i, g] = o[0], l[0], do[0], dl[0]
    return (out, lse), (d_out, d_lse)
