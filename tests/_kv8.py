"""The 8-bit KV cache in 64 bits on the CPU: the definitions of append, attend and evict, written as loops over requests, blocks and
heads, and the error bounds of attention's outputs."""
import math

import numpy as np
import torch

CODES = np.array([math.nan if c & 127 == 127 else
                  (-1.0 if c & 128 else 1.0) * ((1 + (c & 7) / 8) * 2.0 ** ((c >> 3 & 15) - 7) if c >> 3 & 15 else (c & 7) / 8 * 2.0 ** -6)
                  for c in range(256)])
_POSITIVE = CODES[:127]


def nearest_code(x):
    """e4m3 codes of the nearest numbers, ties to the even code, beyond 448 saturated, NaN as 0x7F."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), 448.0)
    hi = np.searchsorted(_POSITIVE, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(x), 127, code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def equal_codes(got, want):
    """Equal bytes, a NaN of either sign equal to the other."""
    ok = (got == want) | ((got & 127 == 127) & (want & 127 == 127))
    if not ok.all():
        i = tuple(np.argwhere(~ok)[0])
        raise AssertionError(f"{(~ok).sum()} of {ok.size} codes differ, first at {i}: {got[i]} for {want[i]}")


def power_for(x):
    """The smallest power of two >= max |x| / 448 over finite x, at least 2^-100."""
    a = np.abs(x[np.isfinite(x)]).max(initial=0.0)
    k = -100
    while 448.0 * 2.0 ** k < a:
        k += 1
    return 2.0 ** k


class Cpu:
    """A cache's contents as numpy arrays: codes [blocks, slots, heads, dim] uint8, scales [blocks, heads]."""

    def __init__(self, k, v, k_scale, v_scale, table):
        self.code = [x.cpu().contiguous().view(torch.uint8).numpy().copy() for x in (k, v)]
        self.scale = [x.cpu().numpy().astype(np.float64) for x in (k_scale, v_scale)]
        self.table = table.cpu().numpy()
        self.bs, self.heads = k.shape[1], k.shape[2]

    def entry(self, row, block):
        e = self.table[row, block]
        return int(e) if 0 <= e < len(self.code[0]) else -1

    def tokens(self, kv, row, n):
        """Values [n, heads, dim]; tokens of blocks outside the cache are None in the second."""
        code = np.zeros((n, self.heads, self.code[0].shape[3]), dtype=np.uint8)
        scale, there = np.ones((n, self.heads)), np.ones(n, dtype=bool)
        for t in range(n):
            e = self.entry(row, t // self.bs)
            if e < 0:
                there[t] = False
                continue
            code[t], scale[t] = self.code[kv][e, t % self.bs], self.scale[kv][e]
        return CODES[code] * scale[:, :, None], there


def append(cache, spans, key, value):
    """spans: (row, start, new, length).  key, value: float64 [total, heads, dim]."""
    for row, start, new, length in spans:
        for block in range(max(length - new, 0) // cache.bs, -(-length // cache.bs)):
            lo, hi = max(length - new, 0, block * cache.bs), min(length, (block + 1) * cache.bs)
            e = cache.entry(row, block)
            if lo >= hi or e < 0:
                continue
            for kv, x in enumerate((key, value)):
                for h in range(cache.heads):
                    fresh = x[start + lo - (length - new):start + hi - (length - new), h]
                    s, slot = power_for(fresh), lo - block * cache.bs
                    if slot:
                        had = cache.scale[kv][e, h]
                        s = max(s, had)
                        if s != had:
                            cache.code[kv][e, :slot, h] = nearest_code(CODES[cache.code[kv][e, :slot, h]] * (had / s))
                    cache.scale[kv][e, h] = s
                    cache.code[kv][e, slot:slot + hi - lo, h] = nearest_code(fresh / s)


U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half a unit in the last place, relative
F = 2.0 ** -24


def attend(cache, spans, q, scale, group, dtype, prior=None, decay=1.0):
    """out, lse, weights {row: [heads, length]}, and for each the largest error allowed.

    Errors: a score is a sum of dim products, each exact, in fp32 (at most dim + 4 roundings of partial sums that are no larger than
    the sum of magnitudes), twice scaled: dz.  p errs by 2 dz (its own score and the maximum's or sum's) and by the roundings of
    exp2 and of a sum of `length` terms.  For its product with V it is rounded to q's type (u), and the result once more (u).
    fp16 loses what lies below 2^-25 of the largest p, and outputs below 2^-25."""
    u, half = U[dtype], dtype == torch.float16
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    d_out, d_lse = np.zeros(q.shape), np.zeros(q.shape[:2])
    weight, d_weight = {}, {}
    dim = q.shape[2]
    for row, start, new, length in spans:
        if length <= 0:
            continue
        (k, there), (v, _) = cache.tokens(0, row, length), cache.tokens(1, row, length)
        w, dw = np.zeros((cache.heads, length)), np.zeros((cache.heads, length))
        for i in range(new):
            seen = (np.arange(length) <= length - new + i) & there
            if not seen.any():
                continue
            for h in range(cache.heads):
                ks, vs = k[seen][:, h], v[seen][:, h]
                for g in range(h * group, (h + 1) * group):
                    x = q[start + i, g]
                    z = ks @ x * scale
                    dz = (dim + 8) * F * float(np.max(np.abs(np.nan_to_num(ks)) @ np.abs(x))) * abs(scale) + 4 * F * float(np.max(np.abs(np.nan_to_num(z))))
                    top = z.max()
                    e = np.exp(z - top)
                    p = e / e.sum()
                    rel = 2 * dz + (len(z) / 4 + 64) * F
                    lse[start + i, g] = top + math.log(e.sum())
                    d_lse[start + i, g] = dz + (len(z) / 4 + 64) * F + 4 * F * abs(lse[start + i, g])
                    out[start + i, g] = p @ vs
                    size = p @ np.abs(vs)
                    d_out[start + i, g] = u * np.abs(out[start + i, g]) + (u + rel) * size
                    if half:
                        d_out[start + i, g] += 2.0 ** -25 * (1 + len(z) * p.max() * np.nanmax(np.abs(vs), initial=0.0))
                    w[h, seen] += p
                    dw[h, seen] += p * rel + 2.0 ** -120
        dw += (new * group + 4) * F * w
        if prior is not None:
            old = decay * prior[row][:, :length - new] if new < length else np.zeros((cache.heads, 0))
            w[:, :old.shape[1]] += old
            dw[:, :old.shape[1]] += 4 * F * (np.abs(old) + w[:, :old.shape[1]])
        weight[row], d_weight[row] = w, dw
    return (out, lse, weight), (d_out, d_lse, d_weight)


def near(got, want, allowed, what):
    got = np.asarray(got, dtype=np.float64)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - want) <= allowed)
    if not ok.all():
        i = tuple(np.argwhere(~ok)[0])
        raise AssertionError(f"{what}: {(~ok).sum()} of {ok.size} off, first at {i}: {got[i]} for {want[i]}, allowed {allowed[i]}")


def evict(cache, spans, weight, to, keep, recent):
    """positions {row: [heads, new length]}; `to` is filled, weights come out as {row: [heads, new length]}."""
    positions, weights = {}, {}
    for row, _, _, length in spans:
        left = min(length, keep)
        positions[row] = np.zeros((cache.heads, left), dtype=np.int64)
        for h in range(cache.heads):
            if length <= keep:
                at = list(range(length))
            else:
                w = [-math.inf if math.isnan(x) else float(x) for x in weight[row][h, :length - recent]]
                at = sorted(sorted(range(length - recent), key=lambda t: (-w[t], t))[:keep - recent]) + list(range(length - recent, length))
            positions[row][h] = at
            for block in range(-(-left // cache.bs)):
                here, e = at[block * cache.bs:(block + 1) * cache.bs], to.entry(row, block)
                if e < 0:
                    continue
                for kv in (0, 1):
                    source = [cache.entry(row, t // cache.bs) for t in here]
                    scales = [cache.scale[kv][b, h] if b >= 0 else 0.0 for b in source]
                    s = max(scales) or 2.0 ** -100
                    to.scale[kv][e, h] = s
                    for slot, (t, b, had) in enumerate(zip(here, source, scales)):
                        to.code[kv][e, slot, h] = nearest_code(CODES[cache.code[kv][b, t % cache.bs, h]] * (had / s)) if b >= 0 else 0
        weights[row] = np.take_along_axis(weight[row][:, :max(length, 1)], positions[row], 1) if left else np.zeros((cache.heads, 0))
    return positions, weights
