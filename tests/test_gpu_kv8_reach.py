"""Kernel variants that only larger calls choose, each with a check that the call chooses it: contexts in several splits while row tiles are
counted on the device, selection past the tokens that a workgroup holds, several blocks moved by a wavefront."""
import math

import numpy as np
import pytest
import torch

import _kv8 as K
from test_gpu_kv8 import B, BF16, DEV, FP16, Setup, _check_attend, _check_evict, _stream        # noqa: F401

pytestmark = pytest.mark.gpu


def _splits(B, s, q_heads, weights):                # noqa: F811
    """Splits of the contexts, out of what the workspace holds: a sum and a maximum, and a row of floats, for each of them."""
    rows = s.total * q_heads
    each = B.kv8_attend_workspace(s.cache, s.batch, q_heads, weights) - (rows * 4 if weights else 0)
    return round(each / (rows * (8 + 4 * s.dim)))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim,weights", [(64, True), (128, True), (128, False), (240, True)])
def test_splits_while_row_tiles_are_counted(B, dtype, dim, weights):                # noqa: F811
    """A prompt among single tokens: by the longest request there would be as many row tiles for each, by all rows there are fewer."""
    heads, group, reqs = 8, 2, 12
    spans = [(1, 5 + 60 * i) for i in range(reqs)]
    spans[7] = (150, 1100)
    s = Setup(B, 51, spans, heads, dim, 16)
    tile = 256 if dim <= 128 else 128
    assert -(-150 * group // tile) * reqs > s.total * group // tile + reqs
    assert _splits(B, s, heads * group, weights) > 1
    _check_attend(B, s, dtype, group, weights=weights)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim", [16, 64, 80, 208])
def test_splits_of_long_parts(B, dtype, dim):       # noqa: F811
    s = Setup(B, 52, [(40, 1700), (33, 600), (3, 90)], 2, dim, 32)
    assert _splits(B, s, 4, True) > 1
    _check_attend(B, s, dtype, 2)


@pytest.mark.parametrize("kind", ["random", "few", "nan"])
@pytest.mark.parametrize("keep,recent", [(100, 30), (8500, 8400), (9000, 0), (1, 0)])
def test_evict_past_the_keys_that_a_workgroup_holds(B, kind, keep, recent):         # noqa: F811
    s = Setup(B, 53, [(0, t) for t in (8192, 8193, 8192 + 512, 9001, 20011)], 1, 16, 64)
    weight = {}
    for row, _, _, t in s.spans:
        x = s.rng.random((1, t)).astype(np.float32) ** 6
        if kind == "few":
            x = np.floor(x * 16).astype(np.float32)
        elif kind == "nan":
            x[s.rng.random((1, t)) > 0.6], x[:, 3], x[:, -40] = math.nan, math.inf, -math.inf
        weight[row] = x
    _check_evict(B, s, keep, recent, weight)


@pytest.mark.parametrize("block,order,spread", [(16, "slots", 3), (32, "heads", 3), (48, "slots", 3), (16, "slots", 30)])
def test_evict_with_several_blocks_a_wavefront(B, block, order, spread):            # noqa: F811
    """64 tokens a wavefront: four blocks of 16, two of 32, one of 48.  Codes, scales and weights, all of them, in 64 bits."""
    heads, dim, reqs, keep, recent = 8, 32, 64, 520, 64
    lens = [int(x) for x in np.random.default_rng(block).integers(1, 700, reqs)]
    lens[0], lens[1], lens[2], lens[3] = 700, 0, keep, keep + 1
    s, to = Setup(B, 54, [(0, t) for t in lens], heads, dim, block, order=order), Setup(B, 55, [(0, keep)] * reqs, heads, dim, block)
    assert min(keep, s.max_len) * reqs * heads >= 64 * 4096
    e = torch.from_numpy(s.rng.integers(-spread, 1, tuple(s.k_scale.shape))).to(DEV)
    s.k_scale.copy_(2.0 ** e.float()), s.v_scale.copy_(2.0 ** (-7.0 - e.float()))
    weight = torch.rand(reqs, heads, s.max_len, device=DEV) ** 6
    positions, new_lens = torch.empty(reqs, heads, keep, dtype=torch.int32, device=DEV), torch.empty(reqs, dtype=torch.int32, device=DEV)
    to_w = torch.full((reqs, heads, keep), 5.0, device=DEV)
    cpu, goal = s.cpu(), to.cpu()
    B.kv8_evict(s.cache, s.batch, weight, to.cache, to_w, keep=keep, recent=recent, positions=positions, lens=new_lens, stream=_stream())
    assert new_lens.tolist() == [min(t, keep) for t in lens]
    w, got_w, got = weight.cpu().numpy(), to_w.cpu().numpy(), positions.cpu().numpy()
    head = np.arange(heads)[:, None]
    for r, length in enumerate(lens):
        left = min(length, keep)
        assert (got[r, :, left:] == -1).all() and (got_w[r, :, left:] == 5.0).all()
        if not left:
            continue
        at = np.broadcast_to(np.arange(left), (heads, left))
        if length > keep:
            old = np.sort(np.argsort(-w[r, :, :length - recent], axis=1, kind="stable")[:, :keep - recent], axis=1)
            at = np.concatenate([old, np.broadcast_to(np.arange(length - recent, length), (heads, recent))], axis=1)
        assert np.array_equal(got[r, :, :left], at)
        assert np.array_equal(got_w[r, :, :left], np.take_along_axis(w[r], at, 1))
        source, target = cpu.table[r][at // block], goal.table[r][np.arange(left) // block]
        for kv in (0, 1):
            had = cpu.scale[kv][source, head]
            now = np.zeros((heads, -(-left // block)))
            np.maximum.at(now, (head, np.broadcast_to(np.arange(left) // block, at.shape)), had)
            goal.scale[kv][goal.table[r][:now.shape[1]]] = now.T
            x = K.CODES[cpu.code[kv][source, at % block, head]] * (had / now[head, np.arange(left) // block])[..., None]
            goal.code[kv][target, np.arange(left) % block] = K.nearest_code(x).transpose(1, 0, 2)
    for x, y in ((to.k, goal.code[0]), (to.v, goal.code[1])):
        K.equal_codes(x.cpu().numpy(), y)
    for x, y in ((to.k_scale, goal.scale[0]), (to.v_scale, goal.scale[1])):
        assert np.array_equal(x.cpu().numpy().astype(np.float64), y, equal_nan=True)
