"""Attention of few query rows over many contexts, cut into equal ranges that pass the ends of requests, and over single long ones in
equal splits: against the definition in 64 bits, as in test_gpu_kv8.py."""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import B, Setup, _check_attend        # noqa: F401

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


def _spans(reqs, new, longest, seed):
    r = np.random.default_rng(seed)
    lens = r.integers(0, 60, reqs)
    lens[[0, reqs // 2, reqs - 1]] = longest, longest // 3, 33
    return [(int(min(new, n)) if i % 5 else 0, int(n)) for i, n in enumerate(lens, 1)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("reqs,heads,group,dim,new,longest", [
    (70, 8, 1, 64, 1, 1500),            # more requests than lanes
    (40, 16, 2, 128, 1, 900),
    (33, 16, 6, 80, 4, 2100),           # two tiles of query rows a wavefront
    (6, 3, 5, 256, 4, 300),             # two wavefronts for a head's query rows
], ids=["many", "some", "wide", "tall"])
@pytest.mark.parametrize("weights", [True, False])
def test_ranges(B, dtype, reqs, heads, group, dim, new, longest, weights):          # noqa: F811
    _check_attend(B, Setup(B, 21, _spans(reqs, new, longest, reqs), heads, dim, 16), dtype, group, weights=weights)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("spans,heads,group,dim", [
    ([(1, 1025), (1, 1), (0, 700)], 1, 4, 64),
    ([(2, 5000), (1, 1200), (3, 3)], 2, 3, 128),
    ([(4, 2500), (4, 40)], 2, 7, 96),   # two tiles of query rows
    ([(1, 3000), (1, 0)], 1, 16, 256),
], ids=["few", "more", "wide", "256"])
@pytest.mark.parametrize("weights", [True, False])
def test_splits(B, dtype, spans, heads, group, dim, weights):                       # noqa: F811
    _check_attend(B, Setup(B, 22, spans, heads, dim, 32), dtype, group, weights=weights)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("reqs,heads,dim,new,longest", [
    (33, 16, 64, 40, 200),              # many more workgroups than compute units
    (70, 8, 80, 34, 150),               # more requests than lanes
    (33, 8, 128, 40, 1100),             # contexts in two splits as well
], ids=["rows", "many", "splits"])
def test_many_rows(B, dtype, reqs, heads, dim, new, longest):                   # noqa: F811
    r = np.random.default_rng(reqs)
    spans = [(int(new if i % 7 else 0), int(n)) for i, n in enumerate(r.integers(new, new + 50, reqs), 1)]
    spans[reqs // 2] = (300, longest + 300)        # a prompt among short ones
    _check_attend(B, Setup(B, 23, spans, heads, dim, 16), dtype, 1)
