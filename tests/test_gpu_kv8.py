"""The operators on the 8-bit KV cache against their definitions in 64 bits: codes, scales, positions and lengths exactly, attention's
outputs within bounds that _kv8.attend derives.  Whatever no request owns is filled with NaN codes and NaN scales."""
import math

import numpy as np
import pytest
import torch

import _kv8 as K

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_2605_11093_amd import binding
    binding.lib()
    return binding


def _stream():
    return torch.cuda.current_stream().cuda_stream


class Setup:
    """A cache with the first `held` tokens of every request in it, and the requests' new ones."""

    def __init__(self, B, seed, spans, heads, dim, block, *, order="slots", seqs=None, room=0, bad=(), fill=True):
        """spans: (new tokens, length) per request; bad: (request, logical block) whose table entry lies outside the cache."""
        rng = np.random.default_rng(seed)
        self.rng, self.n = rng, len(spans)
        seqs = seqs or self.n
        self.rows = list(range(self.n)) if seqs == self.n else sorted(rng.choice(seqs, self.n, replace=False).tolist())
        per = max(1, max(-(-t // block) for _, t in spans)) + room
        blocks = seqs * per + 3
        table = rng.permutation(blocks)[:seqs * per].astype(np.int32).reshape(seqs, per)
        shape = (blocks, block, heads, dim) if order == "slots" else (blocks, heads, block, dim)
        codes = [np.full(shape, 0x7F, dtype=np.uint8) for _ in range(2)]
        scales = [np.full((blocks, heads), np.nan, dtype=np.float32) for _ in range(2)]
        start, self.spans = 0, []
        for r, (new, length) in enumerate(spans):
            self.spans.append((self.rows[r], start, new, length))
            start += new
            held = length if fill else length - new
            for b in range(-(-held // block) if held > 0 else 0):
                e, m = table[self.rows[r], b], min(block, held - b * block)
                for kv in (0, 1):
                    x = np.clip(rng.normal(size=(m, heads, dim)) * 60, -448, 448)
                    c = K.nearest_code(x)
                    codes[kv][e][:m] = c if order == "slots" else 0
                    if order != "slots":
                        codes[kv][e][:, :m] = c.transpose(1, 0, 2)
                    scales[kv][e] = 2.0 ** rng.integers(-7, -4, heads)
        self.total, self.starts = start, [s for _, s, _, _ in self.spans] + [start]
        for r, b in bad:
            table[self.rows[r], b] = blocks + 5 if b % 2 else -1
        self.k, self.v = (torch.from_numpy(c).to(DEV) for c in codes)
        if order != "slots":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.k_scale, self.v_scale = (torch.from_numpy(s).to(DEV) for s in scales)
        self.table = torch.from_numpy(table).to(DEV)
        self.lens = torch.tensor([t for _, _, _, t in self.spans], dtype=torch.int32, device=DEV)
        ones = all(new == 1 for new, _ in spans)
        self.starts_dev = None if ones else torch.tensor(self.starts, dtype=torch.int32, device=DEV)
        self.rows_dev = None if seqs == self.n else torch.tensor(self.rows, dtype=torch.int32, device=DEV)
        self.max_len = max(1, max(t for _, t in spans))
        self.cache = B.KV8(self.k, self.v, self.k_scale, self.v_scale, self.table)
        self.batch = B.KV8Batch(self.lens, starts=self.starts_dev, rows=self.rows_dev, total_new=self.total,
                                max_new=max(1, max(new for new, _ in spans)), max_len=self.max_len)
        self.heads, self.dim, self.seqs, self.per = heads, dim, seqs, per

    def cpu(self):
        return K.Cpu(self.k, self.v, self.k_scale, self.v_scale, self.table)

    def values(self, heads, dtype, spread=1.0):
        x = torch.from_numpy(self.rng.normal(size=(self.total, heads, self.dim)) * spread).to(dtype)
        return x.to(DEV), x.double().numpy()


def _check_attend(B, s, dtype, group, *, weights=True, scale=None, spread=1.3, q=None, decay=0.75, prior=True):
    heads = s.heads * group
    qd, qn = s.values(heads, dtype, spread) if q is None else q
    out = torch.full((s.total, heads, s.dim), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((s.total, heads), 7.0, device=DEV)
    w = p = None
    if weights:
        w = torch.full((s.seqs, s.heads, s.max_len + 3), 5.0, device=DEV)
        p = torch.rand((s.seqs, s.heads, s.max_len + 3), device=DEV) if prior else None
    cpu = s.cpu()
    B.kv8_attend(s.cache, s.batch, qd, out, scale=scale, lse=lse, weight=w, prior=p, decay=decay, stream=_stream())
    spans = [x for x in s.spans if x[3] > 0]
    pn = None if p is None else {row: p[row].cpu().double().numpy() for row, _, _, _ in spans}
    real = scale if scale is not None else s.dim ** -0.5
    (o, l, ww), (do, dl, dw) = K.attend(cpu, spans, qn, real, group, dtype, pn, decay)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")
    if weights:
        got = w.cpu().numpy()
        for row in range(s.seqs):
            if row in ww:
                n = ww[row].shape[1]
                K.near(got[row][:, :n], ww[row], dw[row], f"weight of row {row}")
                assert (got[row][:, n:] == 5.0).all()
            else:
                assert (got[row] == 5.0).all()
    return out, lse, w


ONE = [(1, t) for t in (1, 2, 15, 16, 17, 31, 33, 64, 100, 255, 257, 700)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads,group,dim,block,order", [(2, 4, 128, 16, "slots"), (1, 1, 64, 32, "slots"), (3, 7, 80, 16, "heads"),
                                                         (2, 8, 96, 48, "slots"), (1, 16, 256, 64, "heads"), (1, 33, 16, 16, "slots"),
                                                         (2, 2, 240, 1024, "slots"), (4, 1, 48, 80, "heads")])
def test_attend_single_tokens(B, dtype, heads, group, dim, block, order):
    _check_attend(B, Setup(B, dim + block, ONE, heads, dim, block, order=order, seqs=15), dtype, group)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 4, 128, 16), (1, 1, 64, 32), (2, 3, 80, 16), (1, 7, 96, 48), (1, 2, 256, 64), (1, 5, 16, 16)])
@pytest.mark.parametrize("spans", [[(3, 3), (3, 40), (3, 129)], [(2, 1), (5, 0), (4, 4), (0, 30), (7, 65)],
                                   [(100, 100), (1, 77), (33, 190), (64, 64), (0, 0), (65, 300)]], ids=["three", "ragged", "parts"])
def test_attend_several_tokens(B, dtype, heads, group, dim, block, spans):
    _check_attend(B, Setup(B, 3 * dim + block, spans, heads, dim, block, seqs=len(spans) + 2), dtype, group)


@pytest.mark.parametrize("spans", [[(1, 9000), (1, 3)], [(130, 2500), (1, 1)], [(300, 1500)]], ids=["token", "part", "half"])
def test_attend_long(B, spans):
    _check_attend(B, Setup(B, 5, spans, 2, 128, 16), BF16, 4)


@pytest.mark.parametrize("new", [1, 40])
def test_attend_without_weights_and_with_another_scale(B, new):
    s = Setup(B, 11, [(new, 300), (new, 41)], 2, 64, 16)
    _check_attend(B, s, BF16, 2, weights=False, scale=0.31)
    _check_attend(B, s, BF16, 2, weights=False, scale=-0.2)
    _check_attend(B, s, FP16, 2, prior=False, scale=0.0)


@pytest.mark.parametrize("new", [1, 3, 70])
def test_attend_steep_and_far_scores(B, new):
    """One token takes nearly all of the weight; scores of some thousands."""
    s = Setup(B, 12, [(new, 500), (new, 90)], 2, 128, 16)
    _check_attend(B, s, BF16, 4, spread=60.0)


@pytest.mark.parametrize("new", [1, 3, 50])
def test_attend_blocks_outside_the_cache(B, new):
    s = Setup(B, 13, [(new, 200), (new, 64), (new, new)], 2, 64, 16, bad=[(0, 0), (0, 3), (0, 12), (1, 1), (2, 0), (2, 1 if new > 16 else 0)])
    _check_attend(B, s, BF16, 2)


@pytest.mark.parametrize("new", [1, 4, 90])
def test_attend_nan_in_the_cache(B, new):
    """A NaN in K reaches the queries that see it, one in V the element of the queries that see it, and no others."""
    s = Setup(B, 14, [(new, 150), (new, new)], 2, 64, 16)
    row = s.rows[0]
    t = 149
    block = int(s.table[row, t // 16])
    s.v[block, t % 16, 0, 5] = 0xFF                     # the newest token's V: only the last query sees it
    s.v[int(s.table[row, 1]), 3, 1, 63] = 0x7F
    last = int(s.table[s.rows[1], (new - 1) // 16])
    s.k[last, (new - 1) % 16, 1, 7] = 0x7F              # the newest token's K of the other request
    _check_attend(B, s, BF16, 2, prior=False)


@pytest.mark.parametrize("new", [1, 20])
def test_attend_infinite_and_nan_queries_stay_alone(B, new):
    s = Setup(B, 15, [(new, 100), (new, 60)], 2, 64, 16)
    qd, qn = s.values(4, BF16)
    clean = torch.empty_like(qd)
    B.kv8_attend(s.cache, s.batch, qd, clean, stream=_stream())
    dirty = qd.clone()
    dirty[0, 1, 3], dirty[s.total - 1, 2, 0] = math.nan, math.inf
    out = torch.empty_like(qd)
    B.kv8_attend(s.cache, s.batch, dirty, out, stream=_stream())
    spoiled = torch.zeros(out.shape[:2], dtype=torch.bool, device=DEV)
    spoiled[0, 1] = spoiled[s.total - 1, 2] = True
    assert torch.equal(out[~spoiled], clean[~spoiled])
    assert out[spoiled].isnan().all()


def test_attend_strided_tensors_and_other_streams(B):
    """q, k and v as slices of one projection, outputs inside wider tensors, weights updated in place, on another stream."""
    s = Setup(B, 16, [(5, 90), (1, 33), (40, 45)], 2, 64, 16)
    group, heads = 3, 6
    qd, qn = s.values(heads, BF16)
    wide = torch.full((s.total, heads + 4, 64), math.nan, dtype=BF16, device=DEV)
    wide[:, 2:2 + heads] = qd
    target = torch.full((s.total, heads + 1, 80), 3.0, dtype=BF16, device=DEV)
    w = torch.rand((s.seqs, 2, 100), device=DEV)
    prior = w.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.kv8_attend(s.cache, s.batch, wide[:, 2:2 + heads], target[:, 1:, :64], weight=w, prior=w, decay=0.5, stream=side.cuda_stream)
    side.synchronize()
    pn = {row: prior[row].cpu().double().numpy() for row in s.rows}
    (o, _, ww), (do, _, dw) = K.attend(s.cpu(), s.spans, qn, 64 ** -0.5, group, BF16, pn, 0.5)
    K.near(target[:, 1:, :64].float().cpu().numpy(), o, do, "out")
    for row in s.rows:
        n = ww[row].shape[1]
        K.near(w[row, :, :n].cpu().numpy(), ww[row], dw[row], "weight")
        assert torch.equal(w[row, :, n:], prior[row, :, n:])
    assert (target[:, 0] == 3.0).all() and (target[:, :, 64:] == 3.0).all()


@pytest.mark.parametrize("new", [1, 24])
def test_graph_replays_follow_lengths_and_tables(B, new):
    """A step captured once: appended and attended, replayed with other lengths, tables, tokens; every replay as its eager calls."""
    s = Setup(B, 17, [(new, 200), (new, 70)], 2, 64, 16, room=2)
    key, value, q = torch.empty(s.total, 2, 64, dtype=BF16, device=DEV), torch.empty(s.total, 2, 64, dtype=BF16, device=DEV), \
        torch.empty(s.total, 8, 64, dtype=BF16, device=DEV)
    out, lse, w = torch.empty_like(q), torch.empty(s.total, 8, device=DEV), torch.zeros(2, 2, 240, device=DEV)
    batch = B.KV8Batch(s.lens, starts=s.starts_dev, total_new=s.total, max_new=new, max_len=232)
    work = torch.empty(max(256, B.kv8_attend_workspace(s.cache, batch, 8, True)), dtype=torch.uint8, device=DEV)

    def step():
        B.kv8_append(s.cache, batch, key, value, stream=_stream())
        B.kv8_attend(s.cache, batch, q, out, lse=lse, weight=w, workspace=work, stream=_stream())
    for x in (key, value, q):
        x.copy_(torch.randn_like(x))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    before = [x.clone() for x in (s.k, s.v, s.k_scale, s.v_scale)]
    for i, lens in enumerate([(200, 70), (201, 71), (new, 232), (0, 100)]):
        s.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        s.table.copy_(s.table.roll(i, 1))
        for x in (key, value, q):
            x.copy_(torch.randn_like(x))
        got = []
        for run in (graph.replay, step):
            for x, y in zip((s.k, s.v, s.k_scale, s.v_scale), before):
                x.copy_(y)
            w.zero_()
            run()
            torch.cuda.synchronize()
            got.append([x.clone() for x in (out, lse, w, s.k, s.v, s.k_scale, s.v_scale)])
        for x, y in zip(*got):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_results_do_not_change_from_call_to_call(B):
    s = Setup(B, 18, [(1, 3000), (1, 10), (1, 1500)], 2, 128, 16)
    t = Setup(B, 19, [(200, 1000), (64, 64)], 2, 128, 16)
    for x in (s, t):
        first = None
        q, _ = x.values(8, BF16)
        for _ in range(4):
            out, lse, w = torch.empty_like(q), torch.empty(x.total, 8, device=DEV), torch.zeros(x.seqs, 2, x.max_len, device=DEV)
            B.kv8_attend(x.cache, x.batch, q, out, lse=lse, weight=w, stream=_stream())
            got = [y.view(torch.uint8).clone() for y in (out, lse, w)]
            first = first or got
            assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_contents_that_leave_the_bounds(B):
    """Lengths past max_len, rows outside the table, offsets that run backwards: clamped, and nothing else is touched."""
    s = Setup(B, 20, [(4, 60), (4, 60), (4, 60), (4, 60)], 1, 64, 16)
    qd, qn = s.values(2, BF16)
    lens = torch.tensor([60, 10 ** 6, -5, 60], dtype=torch.int32, device=DEV)
    rows = torch.tensor([0, 1, 2, 9], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 4, 8, 12, 900], dtype=torch.int32, device=DEV)
    batch = B.KV8Batch(lens, starts=starts, rows=rows, total_new=16, max_new=4, max_len=60)
    out, lse, w = torch.full_like(qd, 7.0), torch.full((16, 2), 7.0, device=DEV), torch.full((4, 1, 64), 5.0, device=DEV)
    cpu = s.cpu()
    before = s.k.clone(), s.v.clone()
    key, value = torch.randn(16, 1, 64, device=DEV), torch.randn(16, 1, 64, device=DEV)
    B.kv8_append(s.cache, batch, key, value, stream=_stream())
    K.append(cpu, [(0, 0, 4, 60), (1, 4, 4, 60)], key.double().cpu().numpy(), value.double().cpu().numpy())
    K.equal_codes(s.k.cpu().numpy(), cpu.code[0])
    K.equal_codes(s.v.cpu().numpy(), cpu.code[1])
    for x, y in zip((s.k, s.v), before):
        blocks = s.table[2:].flatten().long()
        assert torch.equal(x[blocks], y[blocks])
    B.kv8_attend(s.cache, batch, qd, out, lse=lse, weight=w, stream=_stream())
    (o, l, _), (do, dl, _) = K.attend(cpu, [(0, 0, 4, 60), (1, 4, 4, 60)], qn, 0.125, 2, BF16)
    K.near(lse.cpu().numpy(), l, dl, "lse")
    K.near(out.float().cpu().numpy(), o, do, "out")
    assert (w[2:] == 5.0).all() and (w[:, :, 60:] == 5.0).all()
    # offsets that run backwards: no new tokens, nothing written
    batch = B.KV8Batch(lens, starts=torch.tensor([9, 4, 3, 2, 1], dtype=torch.int32, device=DEV), rows=rows, total_new=16, max_new=4, max_len=60)
    out.fill_(7.0)
    B.kv8_append(s.cache, batch, key, value, stream=_stream())
    B.kv8_attend(s.cache, batch, qd, out, stream=_stream())
    assert (out == 7.0).all()
    K.equal_codes(s.k.cpu().numpy(), cpu.code[0])
    K.equal_codes(s.v.cpu().numpy(), cpu.code[1])


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("heads,dim,block,order", [(2, 128, 16, "slots"), (3, 80, 32, "heads"), (1, 16, 16, "slots"), (2, 256, 64, "slots"),
                                                   (1, 240, 48, "heads"), (1, 64, 1024, "slots")])
@pytest.mark.parametrize("spans", [[(1, t) for t in (1, 2, 16, 17, 40, 64)], [(3, 3), (0, 20), (50, 50), (5, 2), (17, 33), (130, 140)]],
                         ids=["tokens", "parts"])
def test_append(B, dtype, heads, dim, block, order, spans):
    s = Setup(B, dim, spans, heads, dim, block, order=order, seqs=len(spans) + 1, fill=False)
    key, kn = s.values(heads, dtype, 3.0)
    value, vn = s.values(heads, dtype, 0.2)
    # magnitudes that raise an old scale, and leave it
    for x, n in ((key, kn), (value, vn)):
        for _, start, new, length in s.spans[::2]:
            x[start:start + new] *= 1000
            n[start:start + new] = x[start:start + new].double().cpu().numpy()
    cpu = s.cpu()
    B.kv8_append(s.cache, s.batch, key, value, stream=_stream())
    K.append(cpu, s.spans, kn, vn)
    for got, want in ((s.k, cpu.code[0]), (s.v, cpu.code[1])):
        K.equal_codes(got.cpu().contiguous().numpy(), want)
    for got, want in ((s.k_scale, cpu.scale[0]), (s.v_scale, cpu.scale[1])):
        assert np.array_equal(got.cpu().numpy().astype(np.float64), want, equal_nan=True)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_append_edges(B, dtype):
    """Zeros, subnormals, the type's largest values, infinities and NaN, values on and next to the bounds of a power."""
    s = Setup(B, 1, [(8, 8), (8, 8), (8, 8), (8, 8), (16, 30), (16, 16)], 2, 64, 16, fill=False)
    key, _ = s.values(2, dtype)
    value, _ = s.values(2, dtype)
    big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    key[0:8] = 0
    value[0:8] = tiny / 4
    key[8:16] = torch.linspace(-1, 1, 64, device=DEV).to(dtype) * big
    key[16, 0, 0], key[17, 1, 3], key[18, 0, 2] = math.inf, -math.inf, math.nan
    value[16:24] = math.inf
    value[24:32] = math.nan
    key[24:32] = key[24:32].clamp(-1, 1)
    key[24, 0, 0], key[24, 1, 0] = 448 * 2.0 ** -5, 448 * 2.0 ** -5 * (1 + torch.finfo(dtype).eps)
    cpu = s.cpu()
    B.kv8_append(s.cache, s.batch, key, value, stream=_stream())
    K.append(cpu, s.spans, key.double().cpu().numpy(), value.double().cpu().numpy())
    for got, want in ((s.k, cpu.code[0]), (s.v, cpu.code[1])):
        K.equal_codes(got.cpu().numpy(), want)
    for got, want in ((s.k_scale, cpu.scale[0]), (s.v_scale, cpu.scale[1])):
        assert np.array_equal(got.cpu().numpy().astype(np.float64), want, equal_nan=True)


def test_append_token_by_token_is_near_append_at_once(B):
    """Appended one by one, a block's scale grows; the codes stay within one rounding more of what one call gives."""
    one, many = Setup(B, 2, [(48, 48)], 2, 64, 16, fill=False), Setup(B, 2, [(48, 48)], 2, 64, 16, fill=False)
    key, kn = one.values(2, BF16)
    key *= torch.logspace(-2, 2, 48, base=10, device=DEV, dtype=torch.float32).to(BF16)[:, None, None]
    B.kv8_append(one.cache, one.batch, key, key, stream=_stream())
    cpu = many.cpu()
    for t in range(48):
        lens = torch.tensor([t + 1], dtype=torch.int32, device=DEV)
        B.kv8_append(many.cache, B.KV8Batch(lens, max_len=48), key[t:t + 1], key[t:t + 1], stream=_stream())
        K.append(cpu, [(0, 0, 1, t + 1)], key[t:t + 1].double().cpu().numpy(), key[t:t + 1].double().cpu().numpy())
    K.equal_codes(many.k.cpu().numpy(), cpu.code[0])
    assert torch.equal(many.k_scale.nan_to_num(-1), one.k_scale.nan_to_num(-1))
    a, b = (K.CODES[x.k.cpu().numpy()] * x.k_scale.cpu().double().numpy()[:, None, :, None] for x in (one, many))
    owned = one.table.flatten().tolist()
    step = one.k_scale.cpu().double().numpy()[:, None, :, None] * 2.0 ** -9
    assert (np.abs(a - b)[owned] <= (np.maximum(np.abs(a) * 2.0 ** -3, step))[owned]).all()


def test_append_to_blocks_outside_the_cache(B):
    s = Setup(B, 3, [(40, 40), (1, 17)], 2, 64, 16, fill=False, bad=[(0, 1), (1, 1)])
    key, kn = s.values(2, BF16)
    cpu = s.cpu()
    B.kv8_append(s.cache, s.batch, key, key, stream=_stream())
    K.append(cpu, s.spans, kn, kn)
    K.equal_codes(s.k.cpu().numpy(), cpu.code[0])
    K.equal_codes(s.v.cpu().numpy(), cpu.code[1])


# ------------------------------------------------------------------ evict
def _check_evict(B, s, keep, recent, weight, bad=()):
    to = Setup(B, 77, [(0, keep)] * s.seqs, s.heads, s.dim, s.k.shape[1], bad=bad)
    cpu, goal = s.cpu(), to.cpu()
    w = torch.full((s.seqs, s.heads, s.max_len + 2), math.nan, device=DEV)
    for row, x in weight.items():
        w[row, :, :x.shape[1]] = torch.from_numpy(x).to(DEV)
    to_w = torch.full((s.seqs, s.heads, keep + 1), 5.0, device=DEV)
    positions = torch.full((s.n, s.heads, keep), 9, dtype=torch.int32, device=DEV)
    lens = torch.full((s.n,), 9, dtype=torch.int32, device=DEV)
    B.kv8_evict(s.cache, s.batch, w, to.cache, to_w, keep=keep, recent=recent, positions=positions, lens=lens, stream=_stream())
    want, weights = K.evict(cpu, s.spans, weight, goal, keep, recent)
    assert lens.tolist() == [min(t, keep) for _, _, _, t in s.spans]
    got, got_w = positions.cpu().numpy(), to_w.cpu().numpy()
    for r, (row, _, _, length) in enumerate(s.spans):
        left = min(length, keep)
        assert np.array_equal(got[r][:, :left], want[row]), (r, length)
        assert (got[r][:, left:] == -1).all()
        assert np.array_equal(got_w[row][:, :left], weights[row].astype(np.float32), equal_nan=True)
        assert (got_w[row][:, left:] == 5.0).all()
    for x, y in ((to.k, goal.code[0]), (to.v, goal.code[1])):
        K.equal_codes(x.cpu().numpy(), y)
    for x, y in ((to.k_scale, goal.scale[0]), (to.v_scale, goal.scale[1])):
        assert np.array_equal(x.cpu().numpy().astype(np.float64), y, equal_nan=True)


EVICT = [(0, t) for t in (0, 1, 15, 16, 17, 40, 41, 100, 513, 1100)]


@pytest.mark.parametrize("keep,recent", [(1, 0), (1, 1), (16, 4), (40, 0), (40, 40), (41, 13), (512, 100), (2000, 5)])
@pytest.mark.parametrize("heads,dim,block,order", [(2, 128, 16, "slots"), (1, 80, 32, "heads"), (1, 16, 128, "slots")])
def test_evict(B, keep, recent, heads, dim, block, order):
    s = Setup(B, keep + dim, EVICT, heads, dim, block, order=order, seqs=11)
    weight = {row: s.rng.random((heads, max(t, 1))).astype(np.float32) ** 6 for row, _, _, t in s.spans}
    _check_evict(B, s, keep, recent, weight)


@pytest.mark.parametrize("kind", ["equal", "few", "signs", "nan", "close"])
def test_evict_ties_and_odd_weights(B, kind):
    s = Setup(B, 4, [(0, 700), (0, 90), (0, 1030)], 2, 64, 16)
    weight = {}
    for row, _, _, t in s.spans:
        x = s.rng.random((2, t)).astype(np.float32)
        if kind == "equal":
            x[:] = 0.25
        elif kind == "few":
            x = np.floor(x * 4).astype(np.float32)
        elif kind == "signs":
            x = ((x - 0.5) * 1e-3).astype(np.float32)
            x[:, ::3], x[:, 1::3] = 0.0, -0.0
        elif kind == "nan":
            x[x > 0.5], x[x < 0.1], x[:, 5] = np.nan, -np.inf, np.inf
        else:
            x = (1 + np.floor(x * 8) * 2.0 ** -23).astype(np.float32)
        weight[row] = x
    for keep, recent in ((64, 0), (64, 17), (333, 1)):
        _check_evict(B, s, keep, recent, weight)


def test_evict_blocks_outside_the_caches(B):
    s = Setup(B, 6, [(0, 200), (0, 30)], 2, 64, 16, bad=[(0, 2), (0, 5), (1, 0), (1, 1)])
    weight = {row: s.rng.random((2, t)).astype(np.float32) for row, _, _, t in s.spans}
    _check_evict(B, s, 64, 16, weight, bad=[(0, 1)])


def test_large_offsets(B):
    """A cache whose blocks lie beyond 4 GiB from its base and weights beyond 2^31 bytes: all three operators."""
    heads, dim, block, n = 2, 64, 16, 24
    pitch = 400 << 20
    store = [torch.empty(n * pitch, dtype=torch.uint8, device=DEV) for _ in range(2)]
    k, v = (x.as_strided((n, block, heads, dim), (pitch, heads * dim, dim, 1)) for x in store)
    scales = [torch.ones(n, heads, device=DEV) for _ in range(2)]
    table = torch.randperm(n, device=DEV).to(torch.int32).view(2, 12)
    cache = B.KV8(k, v, *scales, table)
    lens = torch.tensor([150, 96], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 150, 246], dtype=torch.int32, device=DEV)
    batch = B.KV8Batch(lens, starts=starts, total_new=246, max_new=150, max_len=150)
    key, value, q = (torch.randn(246, h, dim, device=DEV, dtype=BF16) for h in (heads, heads, 4))
    w_store = torch.empty(2 * (600 << 20), device=DEV)
    w = w_store.as_strided((2, heads, 150), (600 << 20, 200, 1))
    cpu = K.Cpu(k, v, *scales, table)
    spans = [(0, 0, 150, 150), (1, 150, 96, 96)]
    B.kv8_append(cache, batch, key, value, stream=_stream())
    K.append(cpu, spans, key.double().cpu().numpy(), value.double().cpu().numpy())
    for got, want in ((k, cpu.code[0]), (v, cpu.code[1])):
        got = got.cpu().numpy()
        for row, _, _, t in spans:
            for p in range(t):
                K.equal_codes(got[cpu.entry(row, p // block), p % block], want[cpu.entry(row, p // block), p % block])
    out = torch.empty_like(q)
    B.kv8_attend(cache, batch, q, out, weight=w, stream=_stream())
    (o, _, ww), (do, _, dw) = K.attend(cpu, spans, q.double().cpu().numpy(), 0.125, 2, BF16)
    K.near(out.float().cpu().numpy(), o, do, "out")
    for row, _, _, t in spans:
        K.near(w[row, :, :t].cpu().numpy(), ww[row], dw[row], "weight")
    weight = {row: w[row].cpu().numpy() for row, _, _, _ in spans}
    to_store = [torch.empty(n * pitch, dtype=torch.uint8, device=DEV) for _ in range(2)]
    to = B.KV8(*(x.as_strided((n, block, heads, dim), (pitch, heads * dim, dim, 1)) for x in to_store),
               *(torch.ones(n, heads, device=DEV) for _ in range(2)), table.flip(1).contiguous())
    goal = K.Cpu(to.k, to.v, to.k_scale, to.v_scale, to.block_table)
    positions, lens2 = torch.empty(2, heads, 50, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    B.kv8_evict(cache, batch, w, to, torch.empty(2, heads, 50, device=DEV), keep=50, recent=9, positions=positions, lens=lens2, stream=_stream())
    want, _ = K.evict(cpu, spans, weight, goal, 50, 9)
    for r in range(2):
        assert np.array_equal(positions[r].cpu().numpy(), want[r])
        for p in range(50):
            e = goal.entry(r, p // block)
            K.equal_codes(to.k[e, p % block].cpu().numpy(), goal.code[0][e, p % block])
