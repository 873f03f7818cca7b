"""Attention of few query rows over many contexts, cut into equal ranges that pass the ends of requests, and over single long ones in
equal splits; batches whose requests differ much, whose work is counted on the device: against the definitions in 64 bits, as in
test_gpu_kv8.py."""
import numpy as np
import pytest
import torch

import _kv8 as K
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


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("reqs,heads,dim,block,new", [(70, 3, 80, 16, 200), (9, 2, 128, 32, 700), (130, 1, 64, 16, 400)], ids=["many", "few", "more"])
def test_append_a_prompt_among_short_ones(B, dtype, reqs, heads, dim, block, new):  # noqa: F811
    r = np.random.default_rng(reqs)
    spans = [(int(i % 3 > 0), int(n)) for i, n in enumerate(r.integers(1, 50, reqs))]
    spans[reqs // 3] = (new, new + 21)
    s = Setup(B, 24, spans, heads, dim, block, fill=False)
    key, kn = s.values(heads, dtype, 3.0)
    value, vn = s.values(heads, dtype, 0.2)
    cpu = s.cpu()
    B.kv8_append(s.cache, s.batch, key, value, stream=torch.cuda.current_stream().cuda_stream)
    K.append(cpu, s.spans, kn, vn)
    for got, want in ((s.k, cpu.code[0]), (s.v, cpu.code[1])):
        K.equal_codes(got.cpu().contiguous().numpy(), want)
    for got, want in ((s.k_scale, cpu.scale[0]), (s.v_scale, cpu.scale[1])):
        assert np.array_equal(got.cpu().numpy().astype(np.float64), want, equal_nan=True)
