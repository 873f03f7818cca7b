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
