"""The operators for long contexts on the 8-bit KV cache at the edges of what they accept: scales far from each other, scales that are no
powers of two, queries that are no numbers, no rows, the longest lists; against the definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import _kv8 as K
import _kv8_long as L
from test_gpu_kv8 import B, BF16, DEV, FP16, FP32, Setup, _stream        # noqa: F401
from test_gpu_kv8_edges import _bounds, _scales
import test_gpu_kv8_long as shared
from test_gpu_kv8_long import Shared, _check_blocks, _check_rotated, _check_select, _check_shared, _lists

pytestmark = pytest.mark.gpu


def _same_prefixes(s):
    """Requests' tables begin alike, so their scales do."""
    assert (s.table[s.rows[0], 0] == s.table[s.rows[1], 0]).all()


@pytest.mark.parametrize("groups,group,dim", [
    ([(300, [(1, 310 + i) for i in range(5)])], 4, 64),                         # few rows, the prefix by tokens
    ([(400, [(1, 405 + 9 * i) for i in range(30)])], 4, 128),                   # many rows, the prefix in parts
    ([(190, [(1, 205 + 9 * i) for i in range(30)])], 4, 128),                   # and unsplit
    ([(190, [(40, 250), (33, 300)])], 2, 128),                                  # unsplit under prompts
    ([(100, [(2, 120), (1, 130)])], 4, 256), ([(300, [(50, 350), (3, 320)])], 2, 240)],
    ids=["tokens", "parts", "unsplit", "prompts", "256", "parts240"])
@pytest.mark.parametrize("dtype,kind", [(FP16, "spread"), (FP16, "far"), (FP16, "odd"), (BF16, "odd"), (BF16, "tiny"), (BF16, "wide")])
def test_scales_of_v_behind_prefixes(B, groups, group, dim, dtype, kind):        # noqa: F811
    s = Shared(B, 81, groups, 2, dim, 16)
    _same_prefixes(s)
    s.v_scale.copy_(_scales(s, kind, s.rng))
    if kind == "odd":
        s.k_scale.copy_(_scales(s, kind, s.rng))
    qd, qn = s.values(2 * group, dtype, 1.3)
    out, lse = torch.empty_like(qd), torch.empty(qd.shape[:2], device=DEV)
    B.kv8_attend_shared(s.cache, s.batch, s.prefix, qd, out, lse=lse, stream=_stream())
    (o, l, _), (do, dl, _) = _bounds(s, qn, dim ** -0.5, group, dtype)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")


@pytest.mark.parametrize("dim,length", [(64, 300), (128, 200), (256, 170), (64, 5000)])
@pytest.mark.parametrize("dtype,kind", [(FP16, "spread"), (FP16, "far"), (FP16, "odd"), (BF16, "odd"), (BF16, "tiny"), (BF16, "wide")])
def test_scales_of_v_in_listed_blocks(B, dim, length, dtype, kind):        # noqa: F811
    """Lists of all blocks, the last ones first."""
    s = Setup(B, 82, [(1, length), (1, 40)], 2, dim, 16)
    s.v_scale.copy_(_scales(s, kind, s.rng))
    if kind == "odd":
        s.k_scale.copy_(_scales(s, kind, s.rng))
    n = -(-length // 16)
    lists = np.full((2, 2, n), -1, dtype=np.int32)
    for r, (_, _, _, t) in enumerate(s.spans):
        lists[r, :, :-(-t // 16)] = np.arange(-(-t // 16))[::-1]
    qd, qn = s.values(8, dtype, 1.3)
    out, lse = torch.empty_like(qd), torch.empty(qd.shape[:2], device=DEV)
    B.kv8_attend_blocks(s.cache, s.batch, torch.from_numpy(lists).to(DEV), qd, out, lse=lse, stream=_stream())
    (o, l, _), (do, dl, _) = _bounds(s, qn, dim ** -0.5, 4, dtype)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")


@pytest.mark.parametrize("kind", ["odd", "wide", "tiny"])
def test_selections_by_scales_of_any_size(B, kind):        # noqa: F811
    s = Setup(B, 83, [(1, 16 * 70), (2, 16 * 33)], 2, 64, 16)
    s.k_scale.copy_(_scales(s, kind, s.rng))
    _check_select(B, s, BF16, 3, 20, 1, 1)
    _check_select(B, s, FP16, 3, 20, 1, 1)


def test_rotated_into_blocks_whose_scale_is_no_power_of_two(B):        # noqa: F811
    """Codes are nearest to quotients by the scale that a block has; none of those here lies within fp32's rounding of a border."""
    s = Setup(B, 84, [(5, 21), (1, 4), (20, 45)], 2, 64, 16, fill=False)
    held = s.rng.uniform(1, 2, s.k_scale.shape) * 2.0 ** s.rng.integers(-8, 2, s.k_scale.shape)
    s.k_scale.copy_(torch.from_numpy(held.astype(np.float32)))
    s.v_scale.copy_(torch.from_numpy(held[::-1].astype(np.float32).copy()))
    _check_rotated(B, s, BF16, 4, 64, False)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("many", [False, True])
def test_queries_that_are_no_numbers_spoil_no_others(B, bad, many):        # noqa: F811
    """A query that is no number makes its own output none, and leaves those of other heads and requests alone."""
    s = Shared(B, 85, [(190, [(1, 205 + 9 * i) for i in range(30 if many else 4)])], 2, 128, 16)
    q, qn = s.values(8, BF16)
    clean, spoiled = torch.empty_like(q), torch.empty_like(q)
    B.kv8_attend_shared(s.cache, s.batch, s.prefix, q, clean, stream=_stream())
    q[1, 3, 5] = bad
    B.kv8_attend_shared(s.cache, s.batch, s.prefix, q, spoiled, stream=_stream())
    assert spoiled[1, 3].isnan().any()
    spoiled[1, 3] = clean[1, 3]
    (o, _, _), (do, _, _) = K.attend(s.cpu(), s.spans, qn, 128 ** -0.5, 4, BF16)
    K.near(spoiled.float().cpu().numpy(), o, do, "others")
    blocks = torch.from_numpy(_lists(s, 8)).to(DEV)
    B.kv8_attend_blocks(s.cache, s.batch, blocks, q, spoiled, stream=_stream())
    assert spoiled[1, 3].isnan().any() and spoiled[0].isfinite().all() and spoiled[1, :3].isfinite().all() and spoiled[1, 4:].isfinite().all()


def test_calls_without_rows(B):        # noqa: F811
    """Requests none of which has a new token; a longest length of zero."""
    s = Shared(B, 86, [(32, [(0, 50), (0, 60)])], 2, 64, 16)
    q = torch.empty((0, 8, 64), dtype=BF16, device=DEV)
    for total, most in ((0, 0), (0, 4)):
        batch = B.KV8Batch(s.lens, starts=s.starts_dev, total_new=total, max_new=most, max_len=s.max_len)
        B.kv8_attend_shared(s.cache, batch, s.prefix, q, q, stream=_stream())
        B.kv8_attend_blocks(s.cache, batch, torch.empty((0, 2, 3), dtype=torch.int32, device=DEV), q, q, stream=_stream())
    one = B.KV8Batch(s.lens, max_len=0)
    q, out, lse = torch.ones((2, 8, 64), dtype=BF16, device=DEV), torch.full((2, 8, 64), 7.0, dtype=BF16, device=DEV), torch.zeros(2, 8, device=DEV)
    bounds, blocks = torch.zeros((s.k.shape[0], 2, 2, 64), dtype=torch.uint8, device=DEV), torch.zeros((2, 2, 3), dtype=torch.int32, device=DEV)
    before = s.k.clone()
    B.kv8_append_rotated(s.cache, one, q[:, :2], q[:, :2], B.KV8Rotary(torch.ones(32, device=DEV)), q=q, q_out=out, stream=_stream())
    assert (out == 7.0).all() and torch.equal(before, s.k)
    B.kv8_bound(s.cache, one, bounds, stream=_stream())
    B.kv8_select(s.cache, one, bounds, q, blocks, stream=_stream())
    assert (bounds == 0).all() and (blocks == -1).all()
    for call in (lambda: B.kv8_attend_blocks(s.cache, one, blocks, q, out, lse=lse, stream=_stream()),
                 lambda: B.kv8_attend_shared(s.cache, one, s.prefix, q, out, lse=lse, stream=_stream())):
        out.fill_(7.0)
        call()
        assert (out == 0.0).all() and (lse == -math.inf).all()


def test_one_block_of_everything(B):        # noqa: F811
    """A context of one token and one block, lists and prefixes of one."""
    s = Shared(B, 87, [(1, [(1, 2), (1, 2)])], 1, 16, 16)
    _check_shared(B, s, BF16, 1)
    _check_blocks(B, s, BF16, 1, np.zeros((2, 1, 1), dtype=np.int32))
    _check_select(B, s, BF16, 1, 1, 0, 1)
    s = Setup(B, 88, [(1, 1)], 1, 16, 16, fill=False)
    _check_rotated(B, s, FP32, 1, 16, True)


def test_more_query_heads_than_a_tile(B):        # noqa: F811
    """37 query heads share one: several tiles of rows in prefixes and rests, several sets of rows in selections."""
    s = Shared(B, 89, [(100, [(1, 110 + i) for i in range(4)])], 2, 64, 16)
    _check_shared(B, s, BF16, 37)
    s = Setup(B, 90, [(1, 16 * 40), (2, 16 * 21)], 2, 64, 16)
    _check_select(B, s, BF16, 37, 12, 1, 1)


def test_positions_behind_an_eviction(B):        # noqa: F811
    """Places behind positions, as dmi_kv8_evict leaves them."""
    s = Setup(B, 91, [(1, 120), (1, 90)], 2, 64, 16, fill=False)
    at = [5000, 70000]
    _check_rotated(B, s, BF16, 4, 64, False, positions=at)


@pytest.mark.parametrize("dtype,heads,group,dim,new,kind", [
    (BF16, 16, 4, 128, 1, "spread"), (FP16, 16, 16, 64, 1, "far"), (BF16, 16, 20, 128, 50, "spread"), (FP16, 13, 1, 256, 60, "odd"), (BF16, 16, 32, 80, 50, "tiny")])
def test_lists_of_a_wavefront_each(B, dtype, heads, group, dim, new, kind):        # noqa: F811
    """Many short lists, of one block to all, each gone through by one wavefront."""
    spans = [(1, 17 + 3 * i % 150) for i in range(60)] if new == 1 else [(new, new + 40), (2, 7)]
    s = Setup(B, 92, spans, heads, dim, 16)
    s.v_scale.copy_(_scales(s, kind, s.rng))
    assert s.total * heads >= 768
    _check_blocks(B, s, dtype, group, _lists(s, 5))


@pytest.mark.parametrize("dtype,heads,group,dim", [(BF16, 1, 7, 256), (FP16, 2, 4, 128), (BF16, 1, 24, 64), (FP16, 1, 5, 80)])
@pytest.mark.parametrize("shared,lens", [(50, (900, 1471, 300)), (0, (2000, 64, 1)), (1000, (1010, 2900, 1700))])
def test_many_rows_in_front_of_long_rests_of_unequal_length(B, dtype, heads, group, dim, shared, lens):        # noqa: F811
    """More rows than a tile a head, contexts behind the prefixes (and those of requests without one) in splits that not every request reaches."""
    s = Shared(B, 93, [(shared, [(12, n + 12) for n in lens]), (48, [(1, 60), (9, 700)])], heads, dim, 16, alone=(1, 1))
    _check_shared(B, s, dtype, group)


def _several(B, seed, heads, dim, blocks, block=16, **more):        # noqa: F811
    """Requests with enough tokens for one pass over the bounds to serve several of them; chunks of tokens that end inside of a request, hold
    several of them, a context of a single block and one of many."""
    n = 4300 // heads
    return Setup(B, seed, [(1, 12 * block), (n // 2, n // 2 + 11 * block), (0, 5), (3, blocks * block - 1), (1, 1), (n - n // 2, n - n // 2 + 6 * block)],
                 heads, dim, block, bad=[(1, 4), (5, 3)], **more)


@pytest.mark.parametrize("dtype,heads,group,dim", [(BF16, 32, 1, 64), (FP16, 32, 3, 80), (BF16, 16, 2, 256), (FP16, 32, 8, 16), (BF16, 24, 5, 128)])
def test_selections_of_many_tokens(B, dtype, heads, group, dim):        # noqa: F811
    s = _several(B, 94, heads, dim, 60 if group < 5 else 410, seqs=9)
    _check_select(B, s, dtype, group, 7, 1, 2)
    bounds = np.full((s.k.shape[0], heads, 2, dim), 0x38, dtype=np.uint8)
    bounds[s.rng.integers(0, len(bounds), 9)] = 0x40
    bounds[s.rng.integers(0, len(bounds), 4)] = 0x7F
    _check_select(B, s, dtype, group, 6, 0, 1, bounds=bounds)           # (equal ones, and no numbers)
    _check_select(B, s, dtype, group, 4, 2, 2, bounds=bounds)           # (none by score)


def test_selections_of_many_tokens_whose_scores_lie_close(B):        # noqa: F811
    """Few nearer to each other than fp32 tells apart, and more than there is room for, one token's behind another's."""
    s = Setup(B, 95, [(131, 300), (3, 16 * 301), (2, 16 * 290)], 32, 64, 16)
    s.k_scale.fill_(0.25)
    s.cache = B.KV8(s.k, s.v, s.k_scale, s.v_scale, s.table)
    bounds = np.full((s.k.shape[0], 32, 2, 64), 0x7E, dtype=np.uint8)
    bounds[:, :, :, -1] = s.rng.integers(0, 4, size=bounds.shape[:3])
    q = torch.ones((s.total, 32, 64), dtype=BF16, device=DEV)
    q[..., -1] = 2.0 ** -12
    for _ in range(2):
        _check_select(B, s, BF16, 1, 20, 1, 1, bounds=np.sort(bounds, axis=2), q=(q, q.double().cpu().numpy()))
        bounds[s.rng.random(len(bounds)) < 0.97, :, :, 0] = 0x70


def test_selections_of_many_tokens_of_any_size_and_rows_of_no_request(B):        # noqa: F811
    """Queries far apart, infinite or no number in one pass; rows behind max_new in the middle of a pass are left."""
    s = _several(B, 96, 32, 64, 60)
    most = max(new for _, _, new, _ in s.spans) - 5
    s.batch = B.KV8Batch(s.lens, starts=s.starts_dev, rows=s.rows_dev, total_new=s.total, max_new=most, max_len=s.max_len)
    s.spans = [(row, start, min(new, most), length) for row, start, new, length in s.spans]
    q = torch.from_numpy(s.rng.normal(size=(s.total, 64, 64)) * 2.0 ** s.rng.integers(-125, 110, (s.total, 1, 1))).to(BF16)
    q[5, 3, 2], q[6, 9, 1], q[9, 0] = math.inf, math.nan, 0.0
    _check_select(B, s, BF16, 2, 5, 1, 1, q=(q.to(DEV), q.double().numpy()))


@pytest.mark.parametrize("dtype,heads,group,dim,new,kind", [
    (BF16, 16, 4, 128, 1, "spread"), (FP16, 16, 16, 64, 2, "far"), (BF16, 16, 8, 80, 1, "odd"), (FP16, 16, 1, 256, 3, "tiny")])
@pytest.mark.parametrize("groups", [1, 5])
def test_rests_of_a_wavefront_each(B, dtype, heads, group, dim, new, kind, groups):        # noqa: F811
    """Many requests with few rows and short contexts behind their prefixes, each gone through by one wavefront; some that share nothing."""
    s = Shared(B, 97, [(32 * g + 32, [(new, 32 * g + 32 + new + (i * 7) % 40) for i in range(60 // groups)]) for g in range(groups)], heads, dim, 16, alone=(3, 6))
    assert len(s.spans) * heads > 1024
    s.v_scale.copy_(_scales(s, kind, s.rng))
    qd, qn = s.values(heads * group, dtype, 1.3)
    out, lse = torch.empty_like(qd), torch.empty(qd.shape[:2], device=DEV)
    B.kv8_attend_shared(s.cache, s.batch, s.prefix, qd, out, lse=lse, stream=_stream())
    (o, l, _), (do, dl, _) = _bounds(s, qn, dim ** -0.5, group, dtype)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")


@pytest.mark.parametrize("dtype,heads,group,dim", [(BF16, 1, 2, 128), (BF16, 8, 2, 128), (FP16, 3, 3, 64), (FP16, 8, 3, 64), (BF16, 5, 1, 256), (BF16, 8, 1, 256)])
@pytest.mark.parametrize("groups", [
    [(96, [(300, 400), (2, 150), (70, 240)])],                                  # unsplit, rows that differ much
    [(600, [(90, 700)] * 7)],                                                   # alike, split or not
    [(64, [(150, 220), (3, 90)]), (0, [(40, 60)]), (200, [(33, 240), (1, 201), (260, 470)]), (16, [(9, 30)])]])
def test_row_tiles_by_pairs_and_in_turn(B, dtype, heads, group, dim, groups):        # noqa: F811
    """Eight heads, whose pairs the XCDs have one by one, and other counts, whose row tiles go to them in turn."""
    s = Shared(B, 98, groups, heads, dim, 16, alone=(1, 0))
    _check_shared(B, s, dtype, group)


@pytest.mark.parametrize("call", [
    *(lambda B, d=d, x=x: shared.test_shared_by_single_tokens(B, d, *x)
      for d, x in ((BF16, (2, 4, 64, 16)), (FP16, (1, 7, 80, 32)), (BF16, (2, 1, 256, 16)), (FP16, (2, 8, 128, 16)), (BF16, (1, 32, 96, 48)))),
    lambda B: shared.test_shared_in_splits(B), lambda B: shared.test_shared_by_none(B), lambda B: shared.test_shared_in_place(B),
    lambda B: shared.test_shared_by_requests_that_are_not_there(B), lambda B: shared.test_shared_with_what_is_no_number(B),
    lambda B: shared.test_shared_and_never_split(B, BF16, 128, 4), lambda B: shared.test_shared_and_never_split(B, FP16, 128, 8),
    lambda B: shared.test_shared_by_many_requests_and_groups(B), lambda B: shared.test_shared_by_groups_that_are_none(B, [-5, 2, 1 << 30]),
    *(lambda B, d=d, k=k, x=x: test_scales_of_v_behind_prefixes(B, [(x[0], [(1, x[0] + 9 + 7 * i) for i in range(x[1])])], x[2], x[3], d, k)
      for d, k in ((FP16, "spread"), (FP16, "far"), (FP16, "odd"), (BF16, "tiny")) for x in ((300, 5, 4, 64), (400, 30, 4, 128), (100, 3, 4, 256))),
    *(lambda B, bad=bad: test_queries_that_are_no_numbers_spoil_no_others(B, bad, True) for bad in (math.nan, math.inf))])
def test_prefixes_read_once_for_few_requests(B, monkeypatch, call):        # noqa: F811
    """What short prefixes of few requests are checked for, with bounds that make a launch of their own of them."""
    monkeypatch.setattr(Shared, "READ_ONCE", True)
    call(B)


@pytest.mark.parametrize("once", [False, True])
def test_prefixes_that_the_others_rows_do_not_list(B, monkeypatch, once):        # noqa: F811
    """They are read through the first request's."""
    monkeypatch.setattr(Shared, "READ_ONCE", once)
    s = Shared(B, 99, [(100, [(1, 140), (3, 120), (1, 99 + 16)]), (48, [(1, 50), (1, 90)])], 2, 64, 16, alone=(1, 0))
    q, qn = s.values(8, BF16)
    (o, l, _), (do, dl, _) = K.attend(s.cpu(), s.spans, qn, 64 ** -0.5, 4, BF16)
    for r, n in ((2, 6), (3, 6), (5, 3)):
        s.table[s.rows[r], :n] = -1
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    B.kv8_attend_shared(s.cache, s.batch, s.prefix, q, out, lse=lse, stream=_stream())
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")


@pytest.mark.parametrize("dtype,heads,group,dim,requests,new", [(BF16, 16, 4, 256, 80, 1), (FP16, 32, 1, 128, 90, 1), (BF16, 32, 4, 64, 150, 1), (BF16, 8, 4, 128, 200, 10)])
def test_unsplit_prefixes_that_many_requests_read_once(B, dtype, heads, group, dim, requests, new):        # noqa: F811
    """They go on from the sums of what is behind them; some requests share nothing."""
    s = Shared(B, 100, [(245, [(new, 246 + new + i % 9) for i in range(requests)] + [(1, 30), (0, 250)])], heads, dim, 16, alone=(2, 1))
    _check_shared(B, s, dtype, group)


@pytest.mark.parametrize("dtype,heads,group,dim", [(BF16, 1, 4, 128), (FP16, 2, 7, 64), (BF16, 3, 4, 256), (FP16, 8, 4, 96)])
@pytest.mark.parametrize("in_place", [False, True])
def test_short_prefixes_of_prompts(B, dtype, heads, group, dim, in_place):        # noqa: F811
    """Each prompt reads them by itself, through the first request's row: prefixes of a block, of none, that end inside of a tile, that a request is
    too short for, and what is no number in one."""
    s = Shared(B, 101, [(16, [(20, 40), (90, 106)]), (200, [(40, 240), (130, 330), (33, 190), (0, 210), (1, 201)]), (0, [(50, 50)])], heads, dim, 16, alone=(1, 2))
    s.v[s.table[s.rows[3], 11].item(), 3, 0, 9] = 0x7F
    cpu = s.cpu()
    q, qn = s.values(heads * group, dtype, 1.3)
    for r, n in ((2, 1), (4, 12), (7, 12)):
        s.table[s.rows[r], :n] = -1
    out, lse = q if in_place else torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    B.kv8_attend_shared(s.cache, s.batch, s.prefix, q, out, lse=lse, stream=_stream())
    (o, l, _), (do, dl, _) = K.attend(cpu, s.spans, qn, dim ** -0.5, group, dtype)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")


@pytest.mark.parametrize("path", ["one launch", "two", "several tokens", "more rows than a tile"])
@pytest.mark.parametrize("dtype,size,least,most", [(BF16, 2.0, 104, 121), (FP16, 2.0, 104, 121), (BF16, 2.0 ** 60, 50, 70), (BF16, 2.0 ** -60, -115, -85), (BF16, 2.0 ** -60, -126, -100),
                                                   (FP16, 2.0 ** -10, -126, -110), (BF16, 2.0 ** -45, -126, 120)])
def test_selections_of_scores_past_the_range_of_fp32(B, path, dtype, size, least, most):        # noqa: F811
    """Queries and scales of any size, which 64 bits have room for and fp32 has not; largest scores that are above it among others that are not,
    and nothing but such as are nothing in it.  (Below zero too: those above fp32's range are then the least.)"""
    if path == "several tokens":
        s, group = _several(B, 102, 32, 64, 60), 2
    else:
        s, group = Setup(B, 103, [(1, 16 * (1500 if path == "two" else 90)), (1, 16 * 40)], 1, 64, 16), 20 if path == "more rows than a tile" else 3
    s.k_scale.copy_(torch.from_numpy((2.0 ** s.rng.integers(least, most, s.k_scale.shape)).astype(np.float32)))
    bounds = K.nearest_code(np.sort(s.rng.normal(size=(s.k.shape[0], s.heads, 2, 64)) * 60 + 20, axis=2))
    bounds[s.rng.random(len(bounds)) < 0.1, :, :, 7] = 0x7F
    for sign in (1.0, -1.0):
        q = (torch.from_numpy(np.abs(s.rng.normal(size=(s.total, s.heads * group, 64)))) * (sign * size)).to(dtype)
        for n_select in (7, 36):
            _check_select(B, s, dtype, group, n_select, 1, 1, bounds=bounds, q=(q.to(DEV), q.double().numpy()))


@pytest.mark.parametrize("path", ["one launch", "two", "several tokens"])
def test_selections_write_nothing_behind_their_workspace(B, path):        # noqa: F811
    """Scores of which more lie close to each other than a workgroup has room for go through all of it."""
    if path == "several tokens":
        s = Setup(B, 104, [(131, 300), (3, 16 * 301), (2, 16 * 290)], 32, 64, 16)
    else:
        s = Setup(B, 105, [(1, 16 * (1500 if path == "two" else 400)), (1, 16 * 333)], 2, 64, 16)
    s.k_scale.fill_(0.25)
    bounds = np.full((s.k.shape[0], s.heads, 2, 64), 0x7E, dtype=np.uint8)
    bounds[:, :, :, -1] = np.sort(s.rng.integers(0, 4, size=bounds.shape[:3]), axis=2)
    q = torch.ones((s.total, s.heads, 64), dtype=BF16, device=DEV)
    q[..., -1] = 2.0 ** -12
    need = B.kv8_select_workspace(s.cache, s.batch, 20)
    room = torch.full((need + 8192,), 0x5A, dtype=torch.uint8, device=DEV)
    got = torch.full((s.total, s.heads, 20), 77, dtype=torch.int32, device=DEV)
    want = got.cpu().numpy().copy()
    B.kv8_select(s.cache, s.batch, torch.from_numpy(bounds).to(DEV), q, got, first=1, recent=1, workspace=room[4096:4096 + need], stream=_stream())
    L.select(s.cpu(), s.spans, bounds, q.double().cpu().numpy(), 1, 20, 1, 1, want)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    assert (room[:4096] == 0x5A).all() and (room[4096 + need:] == 0x5A).all()
