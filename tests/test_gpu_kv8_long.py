"""The operators for long contexts on the 8-bit KV cache against their definitions in 64 bits: codes, scales, bounds and selections exactly,
rotated queries and attention's outputs within derived bounds."""
import numpy as np
import pytest
import torch

import _kv8 as K
import _kv8_long as L
from test_gpu_kv8 import B, BF16, DEV, FP16, FP32, Setup, _stream        # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ append, rotated
def _freq(rotary, base=10000.0):
    return torch.tensor([base ** (-2 * i / rotary) for i in range(rotary // 2)], dtype=torch.float32)


def _check_rotated(B, s, dtype, q_heads, rotary, pairs, *, positions=None, fused=False, in_place=False, spread=2.0, spoil=None):    # noqa: F811
    """Appends, and holds codes and scales to the definition exactly, rotated queries to their bound."""
    heads, dim = s.heads, s.dim
    x = torch.from_numpy(s.rng.normal(size=(s.total + 2, q_heads + 2 * heads, dim)) * spread).to(dtype)
    if spoil:
        spoil(x)
    xd = x.to(DEV)
    if fused:
        q, key, value = xd[:, :q_heads], xd[:, q_heads:q_heads + heads], xd[:, q_heads + heads:]
    else:
        q, key, value = (t.contiguous() for t in (xd[:, :q_heads], xd[:, q_heads:q_heads + heads], xd[:, q_heads + heads:]))
    freq = _freq(rotary)
    rot = B.KV8Rotary(freq.to(DEV), positions=None if positions is None else torch.tensor(positions, dtype=torch.int32, device=DEV), pairs=pairs)
    q_out = None if not q_heads else q if in_place else torch.full((s.total + 2, q_heads, dim), 7.0, dtype=dtype, device=DEV)
    before = x[:, :q_heads].double().numpy()
    cpu = s.cpu()
    B.kv8_append_rotated(s.cache, s.batch, key, value, rot, q=q if q_heads else None, q_out=q_out, stream=_stream())
    place = L.places(s.spans, s.total)
    at = [p if p is not None else 0 for p in place] if positions is None else positions[:s.total]
    k, _ = L.rotate(x[:s.total, q_heads:q_heads + heads].double().numpy(), at, freq.numpy(), pairs)
    with np.errstate(over="ignore"):
        k = k.astype(np.float32).astype(np.float64)
    K.append(cpu, s.spans, k, x[:s.total, q_heads + heads:].double().numpy())
    got = s.cpu()
    for kv in (0, 1):
        np.testing.assert_array_equal(got.scale[kv], cpu.scale[kv])
        K.equal_codes(got.code[kv], cpu.code[kv])
    if q_heads:
        y, size = L.rotate(before[:s.total], at, freq.numpy(), pairs)
        out = q_out.double().cpu().numpy()
        for i in range(s.total + 2):
            if i < s.total and place[i] is not None and place[i] >= 0:
                K.near(out[i], y[i], L.rotated_error(y[i], size[i], dtype), f"row {i}")
            else:
                np.testing.assert_array_equal(out[i], before[i] if in_place else 7.0)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("heads,q_heads,dim,rotary,block", [
    (2, 8, 64, 64, 16), (1, 7, 80, 48, 32), (3, 6, 96, 96, 48), (2, 5, 16, 16, 16), (1, 1, 256, 256, 64), (2, 9, 128, 16, 16), (8, 32, 128, 128, 16)])
def test_rotated(B, dtype, pairs, heads, q_heads, dim, rotary, block):        # noqa: F811
    """One token, several, none, those that start inside of a block and end in another."""
    s = Setup(B, 11, [(1, 1), (3, 20), (0, 5), (block + 7, block + 40), (1, 2 * block), (2, 2 * block + 1)], heads, dim, block, fill=False)
    _check_rotated(B, s, dtype, q_heads, rotary, pairs, fused=True)


@pytest.mark.parametrize("block,dim,new", [(256, 256, 300), (1024, 128, 1000), (64, 128, 130), (128, 96, 100)])
def test_rotated_blocks_longer_than_what_a_workgroup_holds(B, block, dim, new):        # noqa: F811
    s = Setup(B, 12, [(new, new + 17), (5, block + 2)], 2, dim, block, fill=False)
    _check_rotated(B, s, BF16, 6, dim, False)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rotated_by_positions(B, dtype):        # noqa: F811
    """Positions of their own: far ones, below zero, the same twice."""
    s = Setup(B, 13, [(4, 30), (1, 17), (3, 3)], 2, 64, 16, fill=False)
    _check_rotated(B, s, dtype, 4, 64, False, positions=[1 << 24, (1 << 30) + 1, -5, 0, 2147483647, 7, 7, 123456789])


def test_rotated_single_tokens_of_many_requests(B):        # noqa: F811
    s = Setup(B, 14, [(1, 1 + 7 * i % 90) for i in range(70)], 2, 128, 16, seqs=75, order="heads", fill=False)
    _check_rotated(B, s, BF16, 8, 128, True)


def test_rotated_one_long_among_single_ones(B):        # noqa: F811
    """Blocks that requests reach are counted on the device."""
    s = Setup(B, 15, [(1, 40 + i) for i in range(40)] + [(400, 430)] + [(1, 3)] * 40, 1, 64, 16, fill=False)
    _check_rotated(B, s, BF16, 3, 32, False, fused=True)


def test_rotated_in_place_and_without_queries(B):        # noqa: F811
    s = Setup(B, 16, [(5, 21), (1, 4)], 2, 80, 16, fill=False)
    _check_rotated(B, s, FP16, 6, 80, False, fused=True, in_place=True)
    s = Setup(B, 17, [(5, 21), (1, 4)], 2, 80, 16, fill=False)
    _check_rotated(B, s, FP16, 0, 80, False)


def test_rotated_what_is_no_number(B):        # noqa: F811
    """A NaN makes its pair NaN and no scale, infinities the largest codes; rows of nothing but such have the least scale."""
    def spoil(x):
        x[0, 4:, 3] = float("nan")
        x[2, 4:, 5] = float("inf")
        x[3, 4:] = float("nan")
        x[5, :4, 1] = -float("inf")
    s = Setup(B, 18, [(4, 4), (3, 40)], 2, 32, 16, fill=False)
    _check_rotated(B, s, BF16, 4, 32, False, spoil=spoil)


def test_rotated_in_places_that_are_not_there(B):        # noqa: F811
    """Blocks outside of the cache are not written (their queries are rotated), more new tokens than a request's length have none in
    front of its first, a row outside of the table is a request of length 0."""
    s = Setup(B, 19, [(3, 20), (20, 40), (5, 3), (2, 18)], 2, 32, 16, bad=[(0, 1), (1, 1)], fill=False)
    _check_rotated(B, s, BF16, 4, 32, False)
    s = Setup(B, 20, [(3, 20), (2, 18)], 2, 32, 16, seqs=3, fill=False)
    s.rows_dev[1] = 77
    s.spans[1] = (0, 3, 2, 0)
    _check_rotated(B, s, BF16, 4, 32, False)


# ------------------------------------------------------------------ bounds
def _check_bound(B, s, order="slots"):        # noqa: F811
    blocks = s.k.shape[0]
    bounds = torch.full((blocks, s.heads, 2, s.dim), 0x55, dtype=torch.uint8, device=DEV)
    want = bounds.cpu().numpy().copy()
    B.kv8_bound(s.cache, s.batch, bounds, stream=_stream())
    L.bound(s.cpu(), s.spans, want)
    got = bounds.cpu().numpy()
    np.testing.assert_array_equal(K.CODES[got], K.CODES[want])
    return bounds


@pytest.mark.parametrize("heads,dim,block,order", [(2, 64, 16, "slots"), (1, 80, 32, "heads"), (3, 256, 64, "slots"), (2, 16, 1024, "heads"),
                                                   (5, 128, 16, "slots"), (2, 112, 48, "slots")])
def test_bounds(B, heads, dim, block, order):        # noqa: F811
    s = Setup(B, 21, [(1, 1), (3, 20), (0, 5), (block + 7, block + 40), (1, 2 * block), (2, 2 * block + 1), (9, 9)], heads, dim, block, order=order, seqs=9,
              bad=[(4, 1)])
    s.k.view(torch.uint8).transpose(1, 2)[s.table[s.rows[3], 0].item(), 0, 3, 1] = 0xFF if order == "slots" else 0x7F      # a NaN of either sign
    s.k[s.table[s.rows[6], 0].item(), :9] = 0x80                                                      # zeros below zero
    _check_bound(B, s)


def test_bounds_one_long_among_single_ones(B):        # noqa: F811
    _check_bound(B, Setup(B, 22, [(1, 40 + i) for i in range(40)] + [(400, 430)] + [(1, 3)] * 40, 3, 64, 16))


# ------------------------------------------------------------------ selections
def _check_select(B, s, dtype, group, n_select, first, recent, *, bounds=None, q=None, spread=1.0):        # noqa: F811
    if bounds is None:
        x = np.sort(s.rng.normal(size=(s.k.shape[0], s.heads, 2, s.dim)) * 60 + 20, axis=2)
        bounds = K.nearest_code(x)
    qd, qn = s.values(s.heads * group, dtype, spread) if q is None else q
    got = torch.full((s.total, s.heads, n_select), 12345, dtype=torch.int32, device=DEV)
    want = got.cpu().numpy().copy()
    B.kv8_select(s.cache, s.batch, torch.from_numpy(bounds).to(DEV), qd, got, first=first, recent=recent, stream=_stream())
    with np.errstate(invalid="ignore", over="ignore"):
        L.select(s.cpu(), s.spans, bounds, qn, group, n_select, first, recent, want)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    return got


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 4, 64, 16), (1, 7, 80, 32), (3, 1, 256, 16), (2, 12, 128, 16), (1, 32, 16, 48)])
def test_selections(B, dtype, heads, group, dim, block):        # noqa: F811
    s = Setup(B, 31, [(1, 1), (1, 9 * block), (1, 9 * block + 1), (1, 20 * block - 1), (1, 8 * block)], heads, dim, block, seqs=7, bad=[(3, 5), (3, 6)])
    for n_select, first, recent in ((8, 1, 2), (1, 0, 1), (5, 4, 1), (30, 2, 2)):
        _check_select(B, s, dtype, group, n_select, first, recent)


def test_selections_of_several_tokens(B):        # noqa: F811
    """Every token has its own: those of a prompt, those behind a context, of requests that have none."""
    s = Setup(B, 32, [(40, 40), (0, 30), (19, 300), (3, 2), (1, 500)], 2, 64, 16)
    _check_select(B, s, BF16, 2, 6, 1, 2)


def test_selections_among_many_blocks(B):        # noqa: F811
    """More than a workgroup keeps, and than one looks up at a time."""
    s = Setup(B, 33, [(1, 16 * 4999 + 3), (1, 16 * 300)], 1, 16, 16)
    _check_select(B, s, BF16, 2, 128, 3, 5)
    _check_select(B, s, BF16, 2, 4500, 3, 5)


def test_selections_of_equal_scores(B):        # noqa: F811
    """The lowest blocks first, whether all are equal or only those at the border; a zero below zero is a zero."""
    s = Setup(B, 34, [(1, 16 * 60), (1, 16 * 33)], 2, 16, 16, bad=[(0, 7)])
    s.k_scale.fill_(0.5)
    s.cache = B.KV8(s.k, s.v, s.k_scale, s.v_scale, s.table)
    bounds = np.zeros((s.k.shape[0], 2, 2, 16), dtype=np.uint8)
    _check_select(B, s, BF16, 2, 12, 2, 3, bounds=bounds)
    bounds[::2] |= 0x80
    _check_select(B, s, BF16, 2, 12, 2, 3, bounds=bounds)
    bounds[s.rng.integers(0, len(bounds), 9)] = 0x38
    _check_select(B, s, BF16, 2, 12, 2, 3, bounds=bounds)


def test_selections_with_what_is_no_number(B):        # noqa: F811
    s = Setup(B, 35, [(1, 16 * 40)], 2, 32, 16)
    x = K.nearest_code(np.sort(s.rng.normal(size=(s.k.shape[0], 2, 2, 32)) * 60, axis=2))
    for j in (3, 9, 11):
        x[s.table[s.rows[0], j].item(), :, :, 4] = 0x7F
    _check_select(B, s, BF16, 2, 30, 1, 1, bounds=x)        # (more places than blocks whose score is a number, by none)
    _check_select(B, s, BF16, 2, 38, 1, 1, bounds=x)
    q, _ = s.values(4, BF16)
    q[0, 1, 3] = float("nan")
    _check_select(B, s, BF16, 2, 30, 1, 1, bounds=x, q=(q, q.double().cpu().numpy()))


@pytest.mark.parametrize("length", [16 * 300, 16 * 1500])
def test_selections_of_scores_that_lie_close(B, length):        # noqa: F811
    """What fp32 cannot tell apart is told apart: scores that differ in the last of some forty bits, and not at all; few of them and
    more than there is room for."""
    s = Setup(B, 37, [(1, length)], 2, 64, 16)
    s.k_scale.fill_(0.25)
    s.cache = B.KV8(s.k, s.v, s.k_scale, s.v_scale, s.table)
    bounds = np.full((s.k.shape[0], 2, 2, 64), 0x7E, dtype=np.uint8)                  # 448
    bounds[:, :, :, -1] = s.rng.integers(0, 4, size=bounds.shape[:3])                 # 0 to 3 * 2^-9
    q = torch.ones((1, 4, 64), dtype=BF16, device=DEV)
    q[..., -1] = 2.0 ** -12
    for _ in range(2):
        _check_select(B, s, BF16, 2, 40, 1, 1, bounds=np.sort(bounds, axis=2), q=(q, q.double().cpu().numpy()))
        some = s.rng.random(len(bounds)) < 0.97
        bounds[some, :, :, 0] = 0x70
    bounds[:] = 0x38
    _check_select(B, s, BF16, 2, 40, 1, 1, bounds=bounds, q=(q, q.double().cpu().numpy()))


@pytest.mark.parametrize("dtype,size", [(FP16, 2.0 ** -22), (FP16, 2.0 ** -14), (BF16, 2.0 ** -120), (BF16, 2.0 ** -132), (BF16, 2.0 ** 118), (BF16, 0.0)])
def test_selections_by_queries_of_any_size(B, dtype, size):        # noqa: F811
    s = Setup(B, 38, [(1, 16 * 90), (1, 16 * 40)], 2, 80, 16)
    q = (torch.from_numpy(s.rng.normal(size=(2, 6, 80))) * size).to(dtype)
    _check_select(B, s, dtype, 3, 20, 1, 1, q=(q.to(DEV), q.double().numpy()))
    if size == 2.0 ** 118:
        q[0, 0, 0], q[1, 3, 3] = float("inf"), -float("inf")
        _check_select(B, s, dtype, 3, 20, 1, 1, q=(q.to(DEV), q.double().numpy()))


def test_no_block_left_out_has_a_larger_score(B):        # noqa: F811
    """Bounds of the codes themselves, and a selection by them: no score of a token in a block is above the block's."""
    s = Setup(B, 36, [(1, 16 * 50)], 1, 64, 16)
    every = B.KV8Batch(s.lens, starts=torch.tensor([0, 800], dtype=torch.int32, device=DEV), total_new=800, max_new=800, max_len=800)
    bounds = torch.zeros((s.k.shape[0], 1, 2, 64), dtype=torch.uint8, device=DEV)
    B.kv8_bound(s.cache, every, bounds, stream=_stream())
    got = _check_select(B, s, BF16, 1, 10, 1, 1, bounds=bounds.cpu().numpy(), q=(q := s.values(1, BF16)))
    k, _ = s.cpu().tokens(0, s.rows[0], 800)
    score = (k[:, 0] @ q[1][0, 0]).reshape(50, 16).max(1)
    b = K.CODES[bounds.cpu().numpy()][s.table[s.rows[0]].cpu().numpy(), 0]
    upper = np.maximum(q[1][0, 0] * b[:, 0], q[1][0, 0] * b[:, 1]).sum(1) * s.cpu().scale[0][s.table[s.rows[0]].cpu().numpy(), 0]
    assert (score <= upper * (1 + 1e-12) + 1e-12).all() and (got[0, 0] >= 0).all()


# ------------------------------------------------------------------ attention over listed blocks
def _check_blocks(B, s, dtype, group, blocks, *, scale=None, q=None, spread=1.3):        # noqa: F811
    heads = s.heads * group
    qd, qn = s.values(heads, dtype, spread) if q is None else q
    out = torch.full((s.total, heads, s.dim), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((s.total, heads), 7.0, device=DEV)
    B.kv8_attend_blocks(s.cache, s.batch, torch.from_numpy(blocks).to(DEV), qd, out, scale=scale, lse=lse, stream=_stream())
    (o, l), (do, dl) = L.attend_blocks(s.cpu(), s.spans, blocks, qn, s.dim ** -0.5 if scale is None else scale, group, dtype)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")
    return out, lse


def _lists(s, n_select, *, order=True):
    """A random choice of blocks for each token and head, its own among them."""
    blocks = np.full((s.total, s.heads, n_select), -1, dtype=np.int32)
    for i, p in enumerate(L.places(s.spans, s.total)):
        if p is None or p < 0:
            continue
        for h in range(s.heads):
            last = p // s.k.shape[1]
            some = s.rng.permutation(last)[:n_select - 1].tolist() + [last]
            blocks[i, h, :len(some)] = sorted(some) if order else some
    return blocks


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 4, 64, 16), (1, 7, 80, 32), (3, 1, 256, 16), (2, 16, 128, 48), (1, 32, 96, 16), (1, 20, 64, 64)])
def test_listed_blocks(B, dtype, heads, group, dim, block):        # noqa: F811
    s = Setup(B, 41, [(1, 1), (1, 9 * block), (3, 9 * block + 1), (1, 20 * block - 1), (2, block + 1), (0, 9), (2, 1)], heads, dim, block, seqs=9, bad=[(3, 5), (3, 6)])
    for n_select in (1, 4, 7, 30):
        _check_blocks(B, s, dtype, group, _lists(s, n_select))


def test_listed_blocks_in_splits(B):        # noqa: F811
    """Few tokens with long lists: several workgroups share one, and leave parts."""
    for dim, dtype, group in ((64, FP16, 4), (128, BF16, 20), (256, BF16, 3)):
        s = Setup(B, 42, [(1, 5000), (2, 3001)], 1, dim, 16, order="heads")
        _check_blocks(B, s, dtype, group, _lists(s, 200))


def test_listed_blocks_in_any_order(B):        # noqa: F811
    """Not in order, one twice, some that are skipped: below 0, behind the token's own, far outside of the table."""
    s = Setup(B, 43, [(1, 500), (4, 320), (1, 40)], 2, 64, 16)
    blocks = _lists(s, 12, order=False)
    blocks[0, 0, 3] = blocks[0, 0, 2]
    blocks[0, 1, 5] = -7
    blocks[1, 0, 4] = 1 << 30
    blocks[2, 1, 2] = 25
    blocks[4, 0] = -1
    _check_blocks(B, s, BF16, 3, blocks)


def test_listed_blocks_with_what_is_no_number(B):        # noqa: F811
    """NaN codes of tokens that a query does not see leave it alone, those that it sees make it NaN."""
    s = Setup(B, 44, [(1, 100), (1, 90), (1, 70)], 1, 64, 16)
    s.v[s.table[s.rows[1], 2].item(), 3, 0, 9] = 0x7F
    s.k[s.table[s.rows[2], 1].item(), 5, 0, 2] = 0xFF
    blocks = _lists(s, 7)
    _check_blocks(B, s, BF16, 4, blocks)
    _check_blocks(B, s, FP16, 4, blocks, scale=-0.3)


def test_listed_blocks_are_what_all_blocks_are(B):        # noqa: F811
    """A selection that leaves nothing out attends as attend does."""
    s = Setup(B, 45, [(3, 200), (1, 129), (40, 40)], 2, 128, 16)
    n = -(-s.max_len // 16)
    blocks = torch.full((s.total, 2, n), -1, dtype=torch.int32, device=DEV)
    q, _ = s.values(8, BF16)
    bounds = torch.zeros((s.k.shape[0], 2, 2, 128), dtype=torch.uint8, device=DEV)
    B.kv8_select(s.cache, s.batch, bounds, q, blocks, stream=_stream())
    out, lse = _check_blocks(B, s, BF16, 4, blocks.cpu().numpy(), q=(q, q.double().cpu().numpy()))
    other, other_lse = torch.empty_like(out), torch.empty_like(lse)
    B.kv8_attend(s.cache, s.batch, q, other, lse=other_lse, stream=_stream())
    assert (out.float() - other.float()).abs().max() <= 2.0 ** -7 * other.float().abs().max()
    torch.testing.assert_close(lse, other_lse, rtol=1e-5, atol=1e-5)


# ------------------------------------------------------------------ shared prefixes
class Shared(Setup):
    """Requests whose rows of the table begin with the blocks of their group's first.  READ_ONCE: the host's bounds are so high that no request
    reads a prefix by itself."""

    READ_ONCE = False

    def __init__(self, B, seed, groups, heads, dim, block, *, alone=(0, 0), **more):        # noqa: F811
        """groups: (shared tokens, [(new tokens, length), ...]); alone: requests in front of the groups and behind them that share nothing."""
        spans = [(1, 20 + i) for i in range(alone[0])] + [x for _, g in groups for x in g] + [(1, 33 + i) for i in range(alone[1])]
        super().__init__(B, seed, spans, heads, dim, block, **more)
        table, at, starts = self.table.cpu().numpy(), alone[0], [alone[0]]
        for shared, g in groups:
            for r in range(at + 1, at + len(g)):
                table[self.rows[r], :shared // block] = table[self.rows[at], :shared // block]
            at += len(g)
            starts.append(at)
        self.table.copy_(torch.from_numpy(table))
        self.group_starts = torch.tensor(starts, dtype=torch.int32, device=DEV)
        self.shared = torch.tensor([shared for shared, _ in groups], dtype=torch.int32, device=DEV)
        longest = max([1] + [shared for shared, _ in groups])
        if self.READ_ONCE:                      # (the table has to be as wide)
            longest = self.max_len = max(self.max_len, (1 << 26) // (self.n * heads * dim) + 2 * block)
            self.batch = B.KV8Batch(self.lens, starts=self.starts_dev, rows=self.rows_dev, total_new=self.total, max_new=max(new for new, _ in spans),
                                    max_len=longest)
            self.table = torch.nn.functional.pad(self.table, (0, -(-longest // block) - self.per), value=-1)
            self.cache = B.KV8(self.k, self.v, self.k_scale, self.v_scale, self.table)
        self.prefix = B.KV8Prefix(self.group_starts, self.shared, max_prefix=longest)


def _check_shared(B, s, dtype, group, *, scale=None, spread=1.3, prefix=None, in_place=False):        # noqa: F811
    heads = s.heads * group
    qd, qn = s.values(heads, dtype, spread)
    out = qd if in_place else torch.full((s.total, heads, s.dim), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((s.total, heads), 7.0, device=DEV)
    B.kv8_attend_shared(s.cache, s.batch, prefix or s.prefix, qd, out, scale=scale, lse=lse, stream=_stream())
    real = scale if scale is not None else s.dim ** -0.5
    (o, l, _), (do, dl, _) = K.attend(s.cpu(), s.spans, qn, real, group, dtype)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 4, 64, 16), (1, 7, 80, 32), (2, 1, 256, 16), (2, 8, 128, 16), (1, 32, 96, 48)])
def test_shared_by_single_tokens(B, dtype, heads, group, dim, block):        # noqa: F811
    """Prefixes that end inside of a block, that are a block, that are nothing; groups of one; requests of no group."""
    s = Shared(B, 51, [(5 * block + 3, [(1, 5 * block + 4 + i) for i in range(9)]), (block, [(1, 3 * block), (1, block + 1)]), (0, [(1, 7), (1, 9)]),
                       (200, [(1, 300)])], heads, dim, block, alone=(2, 3), seqs=25)
    _check_shared(B, s, dtype, group)


@pytest.mark.parametrize("dtype,dim,group", [(BF16, 128, 4), (FP16, 64, 4), (BF16, 256, 2), (FP16, 80, 1)])
def test_shared_by_prompts(B, dtype, dim, group):        # noqa: F811
    """Several new tokens a request, more than 32 rows a head of some."""
    s = Shared(B, 52, [(300, [(40, 340), (3, 310), (0, 305), (90, 400)]), (64, [(1, 65), (64, 128)])], 2, dim, 16, alone=(1, 0))
    _check_shared(B, s, dtype, group)


def test_shared_in_splits(B):        # noqa: F811
    """A long prefix, cut into parts, and long rests, too."""
    s = Shared(B, 53, [(2100, [(1, 2101), (1, 3900), (1, 2150)])], 1, 64, 16, order="heads")
    _check_shared(B, s, BF16, 4)
    _check_shared(B, s, FP16, 4, scale=-0.2)


def test_shared_by_more_than_there_is(B):        # noqa: F811
    """A prefix that reaches into new tokens, or past a request's end, is cut in front of the first of them; a longer one than max_prefix
    counts as that."""
    s = Shared(B, 54, [(64, [(1, 100), (5, 70), (0, 64)])], 2, 64, 16)
    s.shared.fill_(1000)
    _check_shared(B, s, BF16, 4, prefix=B.KV8Prefix(s.group_starts, s.shared, max_prefix=64))
    _check_shared(B, s, BF16, 4, prefix=B.KV8Prefix(s.group_starts, s.shared, max_prefix=40))
    s.shared.fill_(-3)
    _check_shared(B, s, BF16, 4)


def test_shared_by_none(B):        # noqa: F811
    s = Shared(B, 55, [], 2, 64, 16, alone=(3, 0))
    _check_shared(B, s, BF16, 4)


def test_shared_by_requests_that_are_not_there(B):        # noqa: F811
    """A first request whose row lies outside of the table shares nothing; blocks of a prefix that are not there are none for all; a length
    of zero, more new tokens than a length."""
    s = Shared(B, 56, [(64, [(1, 100), (1, 90), (1, 80)])], 2, 64, 16, seqs=4)
    s.rows_dev[0] = -1
    s.spans[0] = (s.rows[0], 0, 1, 0)
    _check_shared(B, s, BF16, 4)
    s = Shared(B, 57, [(64, [(1, 100), (1, 90), (1, 80)])], 2, 64, 16, bad=[(0, 2), (1, 2), (2, 2)])
    _check_shared(B, s, BF16, 4)
    s = Shared(B, 58, [(32, [(1, 50), (1, 0), (3, 2)]), (32, [(2, 60), (2, 70)])], 2, 64, 16)
    _check_shared(B, s, BF16, 4)


def test_shared_with_what_is_no_number(B):        # noqa: F811
    s = Shared(B, 59, [(64, [(1, 100), (1, 90), (6, 80)])], 1, 64, 16)
    s.v[s.table[s.rows[0], 1].item(), 3, 0, 9] = 0x7F
    s.v[s.table[s.rows[1], 5].item(), 3, 0, 7] = 0x7F
    _check_shared(B, s, BF16, 4)
    s.k[s.table[s.rows[0], 2].item(), 3, 0, 9] = 0x7F
    _check_shared(B, s, FP16, 4)


def test_shared_in_place(B):        # noqa: F811
    s = Shared(B, 60, [(64, [(1, 100), (1, 90), (40, 120)])], 2, 64, 16)
    _check_shared(B, s, BF16, 4, in_place=True)


@pytest.mark.parametrize("dtype,dim,group", [(BF16, 128, 4), (FP16, 128, 8), (BF16, 96, 4)])
def test_shared_and_never_split(B, dtype, dim, group):        # noqa: F811
    """Short prefixes under many rows, single tokens and prompts: what is behind them is where their sums begin.  Some requests share
    nothing: of no group, too short for the prefix, without tokens, of a group whose first is too short."""
    s = Shared(B, 62, [(200, [(1, 230 + 7 * i) for i in range(40)] + [(1, 120), (0, 300), (1, 1)])], 2, dim, 16, alone=(3, 2))
    _check_shared(B, s, dtype, group)
    s = Shared(B, 63, [(200, [(40, 300), (3, 210), (50, 120), (90, 400)]), (64, [(3, 40), (64, 128)]), (100, [(20, 200)] * 3)], 2, dim, 16, alone=(1, 1))
    _check_shared(B, s, dtype, group)


def test_rows_behind_max_new_are_left(B):        # noqa: F811
    """A request with more rows than max_new has as many new tokens as that, and the others are no request's."""
    s = Shared(B, 64, [(200, [(40, 300), (30, 290), (40, 280)])], 2, 128, 16)
    batch = B.KV8Batch(s.lens, starts=s.starts_dev, total_new=s.total, max_new=30, max_len=s.max_len)
    q, qn = s.values(8, BF16)
    out, lse = torch.full((s.total, 8, 128), 7.0, dtype=BF16, device=DEV), torch.full((s.total, 8), 7.0, device=DEV)
    B.kv8_attend_shared(s.cache, batch, s.prefix, q, out, lse=lse, stream=_stream())
    spans = [(row, start, 30, length) for row, start, _, length in s.spans]
    (o, l, _), (do, dl, _) = K.attend(s.cpu(), spans, qn, 128 ** -0.5, 4, BF16)
    for start, end in ((30, 40), (100, 110)):
        o[start:end], l[start:end] = 7.0, 7.0
    K.near(out.float().cpu().numpy(), o, do, "out")
    K.near(lse.cpu().numpy(), l, dl, "lse")


def test_shared_by_many_requests_and_groups(B):        # noqa: F811
    """More groups and requests than a wavefront looks at at once."""
    s = Shared(B, 65, [(20 + i % 30, [(1, 52 + (i * k) % 40) for k in range(1 + i % 3)]) for i in range(70)], 1, 64, 16, alone=(2, 5))
    _check_shared(B, s, BF16, 2)
    s = Shared(B, 66, [(40, [(1, 44 + i % 60) for i in range(150)]), (60, [(2, 64 + i) for i in range(5)])], 1, 64, 16)
    _check_shared(B, s, FP16, 4)


@pytest.mark.parametrize("starts", [[3, 1, 0], [0, 100, 200], [-5, 2, 1 << 30], [2, 2, 2]])
def test_shared_by_groups_that_are_none(B, starts):        # noqa: F811
    """Contents that describe no groups lead nowhere: nothing outside of the outputs is written, nothing outside of the tensors read."""
    s = Shared(B, 61, [(64, [(1, 100), (1, 90)]), (64, [(1, 70)])], 2, 64, 16)
    s.group_starts.copy_(torch.tensor(starts, dtype=torch.int32))
    q, _ = s.values(8, BF16)
    out = torch.full((s.total + 1, 8, 64), 7.0, dtype=BF16, device=DEV)
    B.kv8_attend_shared(s.cache, s.batch, s.prefix, q, out[:s.total], stream=_stream())
    torch.cuda.synchronize()
    assert (out[s.total] == 7.0).all()


# ------------------------------------------------------------------ together
def _decode_step(B, s, x, rot, bounds, blocks, out, dense, prefix, ws):        # noqa: F811
    """A step as a serving loop makes it: tokens appended, their blocks' bounds, a selection, attention over it, and over all."""
    st, h = _stream(), s.heads
    q, key, value = x[:, :4 * h], x[:, 4 * h:5 * h], x[:, 5 * h:]
    B.kv8_append_rotated(s.cache, s.batch, key, value, rot, q=q, q_out=ws["q"], stream=st)
    B.kv8_bound(s.cache, s.batch, bounds, stream=st)
    B.kv8_select(s.cache, s.batch, bounds, ws["q"], blocks, first=1, recent=2, workspace=ws["select"], stream=st)
    B.kv8_attend_blocks(s.cache, s.batch, blocks, ws["q"], out, workspace=ws["blocks"], stream=st)
    B.kv8_attend_shared(s.cache, s.batch, prefix, ws["q"], dense, workspace=ws["shared"], stream=st)


@pytest.mark.parametrize("new", [1, 3])
def test_steps_captured_and_replayed(B, new):        # noqa: F811
    """A graph of the whole step, replayed with other lengths, tables and inputs, with eager steps between its replays."""
    s = Shared(B, 71, [(48, [(new, 60 + 30 * i) for i in range(4)]), (32, [(new, 200), (new, 130)])], 2, 64, 16, room=3)
    batch = B.KV8Batch(s.lens, starts=s.starts_dev, total_new=s.total, max_new=new, max_len=s.per * 16)
    s.batch, n_select = batch, 6
    freq, x = _freq(64), torch.zeros((s.total, 12, 64), dtype=BF16, device=DEV)
    rot = B.KV8Rotary(freq.to(DEV))
    bounds = torch.zeros((s.k.shape[0], 2, 2, 64), dtype=torch.uint8, device=DEV)
    blocks = torch.zeros((s.total, 2, n_select), dtype=torch.int32, device=DEV)
    out, dense = (torch.zeros((s.total, 8, 64), dtype=BF16, device=DEV) for _ in range(2))
    need = {"select": B.kv8_select_workspace(s.cache, batch, n_select), "blocks": B.kv8_attend_blocks_workspace(s.cache, batch, 8, n_select),
            "shared": B.kv8_attend_shared_workspace(s.cache, batch, s.prefix, 8)}
    ws = {k: torch.empty(max(v, 1), dtype=torch.uint8, device=DEV) for k, v in need.items()}
    ws["q"] = torch.zeros((s.total, 8, 64), dtype=BF16, device=DEV)
    every = B.KV8Batch(s.lens.clone(), starts=torch.tensor([0] + np.cumsum([t for _, _, _, t in s.spans]).tolist(), dtype=torch.int32, device=DEV),
                       total_new=sum(t for _, _, _, t in s.spans), max_new=s.max_len, max_len=s.max_len)
    B.kv8_bound(s.cache, every, bounds, stream=_stream())
    step = lambda: _decode_step(B, s, x, rot, bounds, blocks, out, dense, s.prefix, ws)        # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        for run in (graph.replay, step):
            spans = [(row, start, n, min(length + (k % 3), s.per * 16)) for row, start, n, length in s.spans]
            s.lens.copy_(torch.tensor([t for _, _, _, t in spans], dtype=torch.int32))
            x.copy_(torch.from_numpy(s.rng.normal(size=x.shape)).to(BF16))
            s.shared[0] = 48 - 16 * (k % 2)
            for t in (out, dense):
                t.fill_(7.0)
            cpu = s.cpu()
            xs = x.double().cpu().numpy()
            run()
            torch.cuda.synchronize()
            place = L.places(spans, s.total)
            key, _ = L.rotate(xs[:, 8:10], place, freq.numpy(), False)
            K.append(cpu, spans, key.astype(np.float32).astype(np.float64), xs[:, 10:])
            got = s.cpu()
            for kv in (0, 1):
                np.testing.assert_array_equal(got.scale[kv], cpu.scale[kv])
                K.equal_codes(got.code[kv], cpu.code[kv])
            y, size = L.rotate(xs[:, :8], place, freq.numpy(), False)
            q = ws["q"].double().cpu().numpy()
            K.near(q, y, L.rotated_error(y, size, BF16), "q")
            want = np.zeros((s.total, 2, n_select), dtype=np.int32)
            L.select(cpu, spans, bounds.cpu().numpy(), q, 4, n_select, 1, 2, want)
            np.testing.assert_array_equal(blocks.cpu().numpy(), want)
            (o, _), (do, _) = L.attend_blocks(cpu, spans, want, q, 0.125, 4, BF16)
            K.near(out.float().cpu().numpy(), o, do, "listed")
            (o, _, _), (do, _, _) = K.attend(cpu, spans, q, 0.125, 4, BF16)
            K.near(dense.float().cpu().numpy(), o, do, "dense")


def test_calls_on_another_stream(B):        # noqa: F811
    s = Shared(B, 72, [(48, [(1, 60 + 30 * i) for i in range(4)])], 2, 64, 16)
    q, qn = s.values(8, BF16)
    out = torch.zeros((s.total, 8, 64), dtype=BF16, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    B.kv8_attend_shared(s.cache, s.batch, s.prefix, q, out, stream=side.cuda_stream)
    side.synchronize()
    (o, _, _), (do, _, _) = K.attend(s.cpu(), s.spans, qn, 0.125, 4, BF16)
    K.near(out.float().cpu().numpy(), o, do, "out")


def test_repeated_calls_are_bit_equal(B):        # noqa: F811
    s = Shared(B, 73, [(1000, [(1, 1010 + 9 * i) for i in range(20)])], 2, 128, 16)
    q, _ = s.values(8, BF16)
    blocks = torch.from_numpy(_lists(s, 30)).to(DEV)
    got = []
    for _ in range(3):
        out, other = torch.zeros((s.total, 8, 128), dtype=BF16, device=DEV), torch.zeros((s.total, 8, 128), dtype=BF16, device=DEV)
        B.kv8_attend_shared(s.cache, s.batch, s.prefix, q, out, stream=_stream())
        B.kv8_attend_blocks(s.cache, s.batch, blocks, q, other, stream=_stream())
        got.append((out, other))
    for x in got[1:]:
        assert torch.equal(x[0], got[0][0]) and torch.equal(x[1], got[0][1])


def test_strided_tensors_and_rows_of_no_request(B):        # noqa: F811
    """Queries, outputs and bounds that lie among others, heads before blocks; total_new past the last request's rows, which stay as they are."""
    s = Shared(B, 74, [(64, [(3, 100 + 40 * i) for i in range(4)])], 2, 80, 16)
    total = s.total + 5
    batch = B.KV8Batch(s.lens, starts=s.starts_dev, total_new=total, max_new=3, max_len=s.max_len)
    wide = torch.from_numpy(s.rng.normal(size=(total, 14, 96))).to(BF16).to(DEV)
    q = wide[:, 3:9, 16:]
    bounds = torch.full((2, s.k.shape[0], 3, 80), 0x55, dtype=torch.uint8, device=DEV).transpose(0, 1)[:, :, :2]
    s2 = s.cpu()
    want = bounds.cpu().numpy().copy()
    B.kv8_bound(s.cache, batch, bounds, stream=_stream())
    L.bound(s2, s.spans, want)
    np.testing.assert_array_equal(K.CODES[bounds.cpu().numpy()], K.CODES[want])
    x = K.nearest_code(np.sort(s.rng.normal(size=want.shape) * 60, axis=2))
    bounds.copy_(torch.from_numpy(x))
    blocks = torch.full((total, 2, 5), 77, dtype=torch.int32, device=DEV)
    lists = np.full((total, 2, 5), 77, dtype=np.int32)
    B.kv8_select(s.cache, batch, bounds, q, blocks, first=1, recent=1, stream=_stream())
    qn = q.double().cpu().numpy()
    L.select(s2, s.spans, x, qn, 3, 5, 1, 1, lists)
    np.testing.assert_array_equal(blocks.cpu().numpy(), lists)
    for call, (o, do) in ((lambda out, lse: B.kv8_attend_blocks(s.cache, batch, blocks, q, out, lse=lse, stream=_stream()),
                           [x[0] for x in L.attend_blocks(s2, s.spans, lists, qn, 80 ** -0.5, 3, BF16)]),
                          (lambda out, lse: B.kv8_attend_shared(s.cache, batch, s.prefix, q, out, lse=lse, stream=_stream()),
                           [x[0] for x in K.attend(s2, s.spans, qn, 80 ** -0.5, 3, BF16)])):
        room = torch.full((total, 14, 96), 7.0, dtype=BF16, device=DEV)
        lse = torch.full((total, 6), 7.0, device=DEV)
        call(room[:, 3:9, 16:], lse)
        got = room.float().cpu().numpy()
        K.near(got[:s.total, 3:9, 16:], o[:s.total], do[:s.total], "out")
        got[:s.total, 3:9, 16:] = 7.0
        assert (got == 7.0).all() and (lse[s.total:] == 7.0).all()


def test_a_cache_past_32_bits(B):        # noqa: F811
    """Blocks that lie more than 2^32 bytes from the first."""
    blocks, heads, dim = (1 << 32) // (16 * 2 * 64) + 40, 2, 64
    k, v = (torch.zeros((blocks, 16, heads, dim), dtype=torch.uint8, device=DEV) for _ in range(2))
    k_scale, v_scale = (torch.ones((blocks, heads), device=DEV) for _ in range(2))
    table = torch.tensor([[blocks - 1 - 3 * i for i in range(12)]], dtype=torch.int32, device=DEV)
    rng = np.random.default_rng(75)
    for c, scale in ((k, k_scale), (v, v_scale)):
        c[table[0].long()] = torch.from_numpy(K.nearest_code(rng.normal(size=(12, 16, heads, dim)) * 60)).to(DEV)
        scale[table[0].long()] = 2.0 ** -6
    cache = B.KV8(k, v, k_scale, v_scale, table)
    batch = B.KV8Batch(torch.tensor([185], dtype=torch.int32, device=DEV), max_len=192)
    few = torch.arange(12, dtype=torch.int32, device=DEV)[None]                       # the same in a cache of its own
    small = B.KV8(*(x[table[0].long()].contiguous() for x in (k, v, k_scale, v_scale)), few)
    x = torch.from_numpy(rng.normal(size=(1, 12, dim))).to(BF16).to(DEV)
    rot = B.KV8Rotary(_freq(dim).to(DEV))
    prefix = B.KV8Prefix(torch.tensor([0, 1], dtype=torch.int32, device=DEV), torch.tensor([100], dtype=torch.int32, device=DEV), max_prefix=100)
    got = []
    for c in (cache, small):
        q, blocks_dev, out, dense = torch.empty_like(x[:, :8]), torch.empty((1, heads, 5), dtype=torch.int32, device=DEV), torch.empty_like(x[:, :8]), torch.empty_like(x[:, :8])
        bounds = torch.zeros((c.k.shape[0], heads, 2, dim), dtype=torch.uint8, device=DEV)
        every = B.KV8Batch(batch.lens, starts=torch.tensor([0, 185], dtype=torch.int32, device=DEV), total_new=185, max_new=185, max_len=192)
        B.kv8_append_rotated(c, batch, x[:, 8:10], x[:, 10:], rot, q=x[:, :8], q_out=q, stream=_stream())
        B.kv8_bound(c, every, bounds, stream=_stream())
        B.kv8_select(c, batch, bounds, q, blocks_dev, first=1, recent=1, stream=_stream())
        B.kv8_attend_blocks(c, batch, blocks_dev, q, out, stream=_stream())
        B.kv8_attend_shared(c, batch, prefix, q, dense, stream=_stream())
        at = c.block_table[0].long()
        got.append([q, blocks_dev, out, dense, c.k[at], c.v[at], c.k_scale[at], c.v_scale[at], bounds[at]])
    for a, b in zip(*got):
        assert torch.equal(a, b)
