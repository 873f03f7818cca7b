"""The operators on the 8-bit KV cache at the edges of what they accept: loose bounds, calls without new tokens, scales far from each other,
queries that are no numbers; against the definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import _kv8 as K
from test_gpu_kv8 import B, BF16, DEV, FP16, Setup, _check_attend, _stream        # noqa: F401

pytestmark = pytest.mark.gpu


def test_bounds_far_above_the_new_tokens(B):        # noqa: F811
    """max_new far above any request's new tokens."""
    s = Setup(B, 36, [(20, 1500), (3, 60), (0, 10)], 8, 64, 16)
    group = 32
    q, _ = s.values(8 * group, BF16)
    got = []
    for most in (20, 1 << 10, 1 << 20, 1 << 24):
        batch = B.KV8Batch(s.lens, starts=s.starts_dev, total_new=s.total, max_new=most, max_len=s.max_len)
        out, lse, w = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV), torch.zeros(3, 8, s.max_len, device=DEV)
        B.kv8_attend(s.cache, batch, q, out, lse=lse, weight=w, stream=_stream())
        got.append((out, lse, w))
    for other in got[1:]:
        for x, y in zip(got[0], other):
            assert (x.float() - y.float()).abs().max() <= 1e-2


@pytest.mark.parametrize("new", [1, 40])
def test_lengths_bounded_by_zero(B, new):        # noqa: F811
    s = Setup(B, 37, [(new, 40), (new, 50)], 2, 64, 16)
    batch = B.KV8Batch(s.lens, starts=s.starts_dev, total_new=s.total, max_new=new, max_len=0)
    q, _ = s.values(4, BF16)
    out, lse, w = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV), torch.full((2, 2, 64), 5.0, device=DEV)
    B.kv8_attend(s.cache, batch, q, out, lse=lse, weight=w, stream=_stream())
    assert (out == 0).all() and (lse == -math.inf).all() and (w == 5.0).all()


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("max_new,max_len", [(0, 90), (1, 90), (64, 90), (64, 2000)])
def test_weights_where_no_request_has_new_tokens(B, in_place, max_new, max_len):        # noqa: F811
    s = Setup(B, 34, [(0, 90), (0, 17), (0, 0)], 2, 64, 16, seqs=5, room=130)
    batch = B.KV8Batch(s.lens, starts=torch.zeros(4, dtype=torch.int32, device=DEV), rows=s.rows_dev, total_new=0, max_new=max_new, max_len=max_len)
    prior = torch.rand(5, 2, max_len, device=DEV)
    w = prior.clone() if in_place else torch.full_like(prior, 5.0)
    want = w.clone()
    for row, _, _, t in s.spans:
        want[row, :, :t] = 0.75 * prior[row, :, :t]
    q = torch.empty(0, 4, 64, dtype=BF16, device=DEV)
    B.kv8_attend(s.cache, batch, q, q, weight=w, prior=w if in_place else prior, decay=0.75, stream=_stream())
    assert torch.equal(w, want)


@pytest.mark.parametrize("new", [1, 40])
def test_queries_in_the_outputs_memory(B, new):        # noqa: F811
    s = Setup(B, 38, [(new, 300), (new, 41)], 2, 64, 16)
    q, _ = s.values(8, BF16)
    out = torch.empty_like(q)
    B.kv8_attend(s.cache, s.batch, q, out, stream=_stream())
    B.kv8_attend(s.cache, s.batch, q, q, stream=_stream())
    assert torch.equal(q, out)


@pytest.mark.parametrize("spans", [[(3, 90), (2, 20)], [(3, 3000), (2, 70)], [(3, 90 + i) for i in range(40)], [(30, 90), (20, 50)], [(40, 1400)]],
                         ids=["whole", "splits", "ranges", "parts", "partsplits"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_weights_of_tokens_that_a_spoiled_query_does_not_see(B, spans, bad):        # noqa: F811
    s = Setup(B, 35, spans, 2, 64, 16)
    q = s.values(8, BF16)
    for _, start, _, _ in s.spans:
        q[0][start, 3, 5], q[1][start, 3, 5] = bad, bad
    _check_attend(B, s, BF16, 4, q=q)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("new", [1, 40])
def test_scale_zero_over_a_block_of_zeros(B, dtype, new):        # noqa: F811
    s = Setup(B, 33, [(new, 100), (new, 45)], 2, 64, 16)
    for row in s.rows:
        for block in range(3):
            e = int(s.table[row, block])
            s.k[e] = 0
            s.k_scale[e] = 2.0 ** -100
    _check_attend(B, s, dtype, 2, scale=0.0, prior=False)


def _bounds(s, q, scale, group, dtype):
    """What _kv8.attend gives, but fp16's own bound token by token: a p below fp16's normal numbers is off by 2^-25 at most, and by no more
    than itself, times that token's V; an output below them by 2^-25."""
    (o, l, w), (do, dl, dw) = K.attend(s.cpu(), s.spans, q, scale, group, BF16)
    if dtype == BF16:
        return (o, l, w), (do, dl, dw)
    cpu, do = s.cpu(), np.zeros_like(do)
    for row, start, new, length in s.spans:
        if length <= 0:
            continue
        (k, there), (v, _) = cpu.tokens(0, row, length), cpu.tokens(1, row, length)
        for i in range(new):
            seen = (np.arange(length) <= length - new + i) & there
            if not seen.any():
                continue
            for g in range(q.shape[1]):
                ks, vs = k[seen][:, g // group], np.abs(v[seen][:, g // group])
                z = ks @ q[start + i, g] * scale
                p = np.exp(z - z.max())
                p /= p.sum()
                dz = (s.dim + 8) * K.F * float(np.max(np.abs(ks) @ np.abs(q[start + i, g]))) * abs(scale) + 4 * K.F * float(np.abs(z).max())
                rel = 2 * dz + (len(z) / 4 + 64) * K.F
                u = K.U[FP16]
                do[start + i, g] = u * np.abs(o[start + i, g]) + (u + rel) * (p @ vs) + np.minimum(p, 2.0 ** -25) @ vs + 2.0 ** -25
    return (o, l, w), (do, dl, dw)


def _scales(s, kind, rng):
    blocks = s.v_scale.shape
    if kind == "spread":
        e = rng.integers(-14, 3, blocks)
    elif kind == "far":
        e = np.where(rng.random(blocks) < 0.5, -26, 1)
    elif kind == "tiny":
        e = rng.integers(-118, -100, blocks)
    elif kind == "wide":
        e = rng.integers(-70, 30, blocks)
    else:
        e = rng.integers(-7, -4, blocks)
    x = 2.0 ** e
    if kind == "odd":
        x = x * rng.uniform(1, 2, blocks)
    return torch.from_numpy(x.astype(np.float32)).to(DEV)


@pytest.mark.parametrize("spans,group,dim", [
    ([(1, 300), (1, 40)], 4, 128), ([(3, 200), (3, 33)], 2, 64), ([(1, 3000)], 4, 64), ([(4, 150), (2, 70)], 7, 80), ([(1, 200), (1, 17)], 4, 256),
    ([(40, 150), (33, 70)], 2, 64), ([(50, 300), (5, 120)], 2, 128), ([(20, 90), (60, 60)], 2, 240), ([(40, 1300)], 2, 128)],
    ids=["token", "some", "splits", "wide", "256", "parts64", "parts128", "parts240", "partsplits"])
@pytest.mark.parametrize("dtype,kind", [(FP16, "spread"), (FP16, "far"), (FP16, "odd"), (BF16, "spread"), (BF16, "odd"), (BF16, "tiny"), (BF16, "wide")])
def test_scales_of_v(B, spans, group, dim, dtype, kind):        # noqa: F811
    s = Setup(B, 31, spans, 2, dim, 16)
    s.v_scale.copy_(_scales(s, kind, s.rng))
    if kind == "odd":
        s.k_scale.copy_(_scales(s, kind, s.rng))
    qd, qn = s.values(2 * group, dtype, 1.3)
    out, lse = torch.empty_like(qd), torch.empty(qd.shape[:2], device=DEV)
    w = torch.zeros(s.seqs, 2, s.max_len, device=DEV)
    B.kv8_attend(s.cache, s.batch, qd, out, lse=lse, weight=w, stream=_stream())
    (o, l, ww), (do, dl, dw) = _bounds(s, qn, dim ** -0.5, group, dtype)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")
    for row, _, _, t in s.spans:
        K.near(w[row, :, :t].cpu().numpy(), ww[row], dw[row], "weight")


@pytest.mark.parametrize("new", [1, 3, 50])
@pytest.mark.parametrize("dtype", [FP16, BF16])
def test_a_loud_block_of_no_weight(B, new, dtype):        # noqa: F811
    s = Setup(B, 32, [(new, 400), (new, 100)], 2, 128, 16)
    s.v_scale.copy_(_scales(s, "", s.rng))
    for r, block in ((0, 3), (0, 20), (1, 5)):
        e = int(s.table[s.rows[r], block])
        s.k[e] = int(K.nearest_code(-200.0))
        s.v_scale[e] = 2.0 ** 8
    qd, qn = s.values(8, dtype, 1.3)
    qd, qn = qd.abs(), np.abs(qn)
    out = torch.empty_like(qd)
    B.kv8_attend(s.cache, s.batch, qd, out, stream=_stream())
    (o, _, _), (do, _, _) = _bounds(s, qn, 128 ** -0.5, 4, dtype)
    K.near(out.float().cpu().numpy(), o, do, "out")


@pytest.mark.parametrize("dtype", [FP16, BF16])
@pytest.mark.parametrize("spans,heads", [([(33, 1090 + 7 * i) for i in range(16)], 16), ([(1, 9000)], 2), ([(2, 2000 + i) for i in range(20)], 8)],
                         ids=["parts", "splits", "ranges"])
def test_scales_of_v_that_drift(B, dtype, spans, heads):        # noqa: F811
    """From 2^-30 to 2^4 and back over a long context."""
    s = Setup(B, 41, spans, heads, 64, 16)
    for row, _, _, length in s.spans:
        blocks = -(-length // 16)
        e = np.round(-13 + 17 * np.sin(np.arange(blocks) / 6.0)).astype(int)
        s.v_scale[s.table[row, :blocks].long()] = torch.from_numpy(2.0 ** e).float().to(DEV)[:, None].expand(blocks, heads)
    qd, qn = s.values(heads, dtype, 1.3)
    out, lse = torch.empty_like(qd), torch.empty(qd.shape[:2], device=DEV)
    B.kv8_attend(s.cache, s.batch, qd, out, lse=lse, stream=_stream())
    (o, l, _), (do, dl, _) = _bounds(s, qn, 64 ** -0.5, 1, dtype)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")


def test_evict_with_blocks_that_lie_backwards(B):        # noqa: F811
    """block_stride and head_stride below zero, in both caches."""
    s, to = Setup(B, 39, [(0, 200), (0, 30)], 2, 64, 16), Setup(B, 40, [(0, 64)] * 2, 2, 64, 16)
    weight = torch.rand(2, 2, 200, device=DEV)

    def call(cache, dst):
        positions, lens = torch.empty(2, 2, 64, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
        to_w = torch.zeros(2, 2, 64, device=DEV)
        B.kv8_evict(cache, s.batch, weight, dst, to_w, keep=64, recent=9, positions=positions, lens=lens, stream=_stream())
        return positions, lens, to_w

    def backwards(x):
        """The same blocks and heads in memory in the other order; element (0, 0, 0, 0) is the last block's last head."""
        k, v = (y.flip(0, 2).contiguous() for y in (x.k, x.v))
        c = B.KV8(k, v, x.k_scale, x.v_scale, x.table)
        at = (k.shape[0] - 1) * k.stride(0) + (k.shape[2] - 1) * k.stride(2)
        c._raw = B._PACK_KV8(k.data_ptr() + at, v.data_ptr() + at, x.k_scale.data_ptr(), x.v_scale.data_ptr(), -k.stride(0), k.stride(1), -k.stride(2),
                             x.k_scale.stride(0), x.k_scale.stride(1), k.shape[1], k.shape[2], k.shape[3], k.shape[0], x.table.shape[0],
                             x.table.shape[1], x.table.data_ptr(), x.table.stride(0))
        return c, k, v
    c, _, _ = backwards(s)
    t, tk, tv = backwards(to)
    scales = to.k_scale.clone(), to.v_scale.clone()
    got = call(c, t)
    got_scales = to.k_scale.clone(), to.v_scale.clone()
    to.k_scale.copy_(scales[0]), to.v_scale.copy_(scales[1])
    want = call(s.cache, to.cache)
    for x, y in zip((*got, *got_scales), (*want, to.k_scale, to.v_scale)):
        assert torch.equal(x.nan_to_num(-1), y.nan_to_num(-1))
    assert torch.equal(tk.flip(0, 2), to.k) and torch.equal(tv.flip(0, 2), to.v)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("spans,group", [([(5, 3), (4, 0), (3, 40)], 4), ([(60, 30), (40, 0), (50, 50), (33, 1)], 2), ([(64, 1400), (80, 20)], 2)],
                         ids=["few", "many", "splits"])
def test_more_new_tokens_than_the_length(B, dtype, spans, group):        # noqa: F811
    """The first of them have no position: they see nothing, and are not stored."""
    s = Setup(B, 42, spans, 2, 64, 16)
    _check_attend(B, s, dtype, group)
    s = Setup(B, 43, spans, 2, 64, 16, fill=False)
    (key, kn), (value, vn) = s.values(2, dtype, 3.0), s.values(2, dtype, 0.2)
    cpu = s.cpu()
    B.kv8_append(s.cache, s.batch, key, value, stream=_stream())
    K.append(cpu, s.spans, kn, vn)
    for got, want in ((s.k, cpu.code[0]), (s.v, cpu.code[1])):
        K.equal_codes(got.cpu().numpy(), want)


@pytest.mark.parametrize("new", [3, 40])
def test_a_scale_that_takes_a_hidden_code_past_the_largest_number(B, new):        # noqa: F811
    """bf16 holds no 448 * 2^120; a query that does not see it is none the worse, and one that sees smaller codes there has them."""
    s = Setup(B, 44, [(new, 200), (new, 80)], 2, 64, 16)
    for r, length in ((0, 200), (1, 80)):
        e = int(s.table[s.rows[r], (length - 1) // 16])
        s.v_scale[s.table[s.rows[r]].long()] = 2.0 ** 100
        s.v_scale[e] = 2.0 ** 120
        s.v[e] = int(K.nearest_code(2.0 ** -6))
        s.v[e, (length - 1) % 16, 1] = 0x7E
    qd, qn = s.values(4, BF16)
    out = torch.empty_like(qd)
    B.kv8_attend(s.cache, s.batch, qd, out, stream=_stream())
    (o, _, _), (do, _, _) = K.attend(s.cpu(), s.spans, qn, 0.125, 2, BF16)
    for row, start, _, _ in s.spans:
        K.near(out[start:start + new - 1].float().cpu().numpy(), o[start:start + new - 1], do[start:start + new - 1], "out")
        K.near(out[start:start + new, :2].float().cpu().numpy(), o[start:start + new, :2], do[start:start + new, :2], "out")
