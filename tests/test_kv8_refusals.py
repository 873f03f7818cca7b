"""What the operators on the 8-bit KV cache refuse before any GPU work, and the CPU definitions that their tests use."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import _kv8 as K
from paper_2605_11093_amd import binding as B


def _cache(blocks=8, block=16, heads=2, dim=64, seqs=2, wide=4, dtype=torch.uint8):
    k = torch.zeros(blocks, block, heads, dim, dtype=dtype)
    return B.KV8(k, k.clone(), torch.ones(blocks, heads), torch.ones(blocks, heads), torch.zeros(seqs, wide, dtype=torch.int32))


def _batch(n=2, max_len=32, **more):
    return B.KV8Batch(torch.ones(n, dtype=torch.int32), max_len=max_len, **more)


def _q(n=2, heads=4, dim=64, dtype=torch.bfloat16):
    return torch.zeros(n, heads, dim, dtype=dtype)


def _refused(call, *words):
    with pytest.raises((B.DmiError, ValueError)) as e:
        call()
    if isinstance(e.value, B.DmiError):
        assert e.value.code == B.ERR_INVALID_ARG
    for w in words:
        assert w in str(e.value), str(e.value)


def test_cache_shapes():
    for more, word in (({"block": 24}, "block_size"), ({"block": 1040}, "block_size"), ({"dim": 72}, "head_dim"), ({"dim": 272}, "head_dim")):
        c = _cache(**more)
        _refused(lambda: B.kv8_append(c, _batch(), *(torch.zeros(2, 2, c.head_dim),) * 2), *([word] if "dim" not in more or c.head_dim % 16 == 0 else []))
    _refused(lambda: B.KV8(torch.zeros(4, 16, 2, 64), torch.zeros(4, 16, 2, 64), torch.ones(4, 2), torch.ones(4, 2), torch.zeros(1, 4, dtype=torch.int32)), "k must")
    k = torch.zeros(4, 16, 2, 64, dtype=torch.uint8)
    _refused(lambda: B.KV8(k, k, torch.ones(4, 3), torch.ones(4, 3), torch.zeros(1, 4, dtype=torch.int32)), "scales")
    _refused(lambda: B.KV8(k, k.transpose(1, 2).contiguous().transpose(1, 2), torch.ones(4, 2), torch.ones(4, 2), torch.zeros(1, 4, dtype=torch.int32)), "share")
    _refused(lambda: B.KV8(k, k, torch.ones(4, 2), torch.ones(4, 2), torch.zeros(1, 4, dtype=torch.int64)), "block_table")


def test_alignment():
    base = torch.zeros(4 * 16 * 2 * 64 + 64, dtype=torch.uint8)
    k = base[8:8 + 4 * 16 * 2 * 64].view(4, 16, 2, 64)
    at = (-base.data_ptr()) % 16 + 8
    k = base[at:at + 4 * 16 * 2 * 64].view(4, 16, 2, 64)
    c = B.KV8(k, k, torch.ones(4, 2), torch.ones(4, 2), torch.zeros(2, 4, dtype=torch.int32))
    _refused(lambda: B.kv8_append(c, _batch(), *(torch.zeros(2, 2, 64),) * 2), "16-byte aligned")
    odd = torch.zeros(2, 5, 72, dtype=torch.bfloat16)[:, :4, 4:68]
    _refused(lambda: B.kv8_attend(_cache(), _batch(), odd, _q()), "q must be 16-byte")
    _refused(lambda: B.kv8_attend(_cache(), _batch(), _q(), odd), "out must be 16-byte")
    _refused(lambda: B.kv8_attend(_cache(), _batch(), torch.zeros(2, 4, 68, dtype=torch.bfloat16)[:, :, :64].as_strided((2, 4, 64), (275, 68, 1)), _q()), "q must be")


def test_batches():
    c = _cache()
    x = torch.zeros(2, 2, 64)
    _refused(lambda: B.kv8_append(c, _batch(max_len=65), x, x), "max_len")
    _refused(lambda: B.kv8_append(c, _batch(n=3), torch.zeros(3, 2, 64), torch.zeros(3, 2, 64)), "n_reqs")
    _refused(lambda: _batch(starts=torch.zeros(3, dtype=torch.int32)), "total_new")
    _refused(lambda: _batch(starts=torch.zeros(2, dtype=torch.int32), total_new=2), "starts")
    _refused(lambda: _batch(rows=torch.zeros(3, dtype=torch.int32)), "rows")
    _refused(lambda: B.kv8_append(c, _batch(total_new=1), x, x), "one new token")
    _refused(lambda: B.kv8_append(c, _batch(max_new=2), x, x), "one new token")
    _refused(lambda: B.KV8Batch(torch.ones(2), max_len=3), "lens")


def test_append():
    c = _cache()
    x = torch.zeros(2, 2, 64)
    _refused(lambda: B.kv8_append(c, _batch(), x, x.half()), "dtype")
    _refused(lambda: B.kv8_append(c, _batch(), x[:, :1], x), "key must")
    _refused(lambda: B.kv8_append(c, _batch(), x, x[:1]), "value must")


def test_attend():
    c, b = _cache(), _batch()
    _refused(lambda: B.kv8_attend(c, b, _q(heads=3), _q(heads=3)), "query heads")
    _refused(lambda: B.kv8_attend(c, b, _q(dtype=torch.float32), _q(dtype=torch.float32)), "BF16")
    _refused(lambda: B.kv8_attend(c, b, _q(), _q(dtype=torch.float16)), "both")
    _refused(lambda: B.kv8_attend(c, b, _q(), _q(n=1)), "out must")
    _refused(lambda: B.kv8_attend(c, b, _q(dim=48), _q()), "q must")
    _refused(lambda: B.kv8_attend(c, b, _q(), _q(), scale=math.inf), "scale")
    _refused(lambda: B.kv8_attend(c, b, _q(), _q(), lse=torch.zeros(2, 3)), "lse")
    _refused(lambda: B.kv8_attend(c, b, _q(), _q(), lse=torch.zeros(2, 4, dtype=torch.float16)), "lse")
    _refused(lambda: B.kv8_attend(c, b, _q(), _q(), prior=torch.zeros(2, 2, 32)), "prior")
    _refused(lambda: B.kv8_attend(c, b, _q(), _q(), weight=torch.zeros(2, 2, 31)), "weight")
    w = torch.zeros(2, 2, 32)
    _refused(lambda: B.kv8_attend(c, b, _q(), _q(), weight=w, prior=w, decay=math.nan, workspace=torch.zeros(1 << 16, dtype=torch.uint8)), "decay")
    need = B.kv8_attend_workspace(c, b, 4, True)
    assert need > 0
    _refused(lambda: B.kv8_attend(c, b, _q(), _q(), weight=w, workspace=torch.zeros(need - 1, dtype=torch.uint8)), "workspace")


def test_evict():
    c, b, w = _cache(), _batch(), torch.zeros(2, 2, 32)

    def call(keep=16, recent=4, to=None, positions=None, lens=None, weight=w, to_weight=w):
        B.kv8_evict(c, b, weight, to or _cache(), to_weight, keep=keep, recent=recent,
                    positions=torch.zeros(2, 2, keep, dtype=torch.int32) if positions is None else positions,
                    lens=torch.zeros(2, dtype=torch.int32) if lens is None else lens)
    _refused(lambda: call(keep=0, recent=0), "keep")
    _refused(lambda: call(recent=17), "recent")
    _refused(lambda: call(keep=65), "keep")
    _refused(lambda: call(to=_cache(dim=80)), "differ")
    _refused(lambda: call(to=_cache(block=32)), "differ")
    _refused(lambda: call(to=_cache(seqs=1)), "rows")
    _refused(lambda: call(positions=torch.zeros(2, 2, 15, dtype=torch.int32)), "positions")
    _refused(lambda: call(lens=torch.zeros(3, dtype=torch.int32)), "lens")
    _refused(lambda: call(lens=b.lens), "lens_dev")
    _refused(lambda: call(weight=w[:, :1]), "weight")
    _refused(lambda: call(weight=w.double()), "weight")
    _refused(lambda: call(to_weight=torch.zeros(2, 2, 15)), "to_weight")


def test_null_pointers_and_struct_sizes():
    L = B.lib()
    c, b = _cache(), _batch()
    assert len(c._raw) == 112 and len(b._raw) == 40
    for args in ((None, b._raw), (c._raw, None)):
        assert L.dmi_kv8_append(*args, None, None, None) == B.ERR_INVALID_ARG
        assert L.dmi_kv8_attend(*args, None, 4, 1.0, None, None, None, None, 0.0, None, 0, None) == B.ERR_INVALID_ARG
        assert L.dmi_kv8_evict(*args, None, None, None, 1, 1, None, None, None) == B.ERR_INVALID_ARG
        assert L.dmi_kv8_attend_workspace(*args, 4, 1) == 0
    assert L.dmi_kv8_append(c._raw, b._raw, None, None, None) == B.ERR_INVALID_ARG
    assert b"NULL" in L.dmi_last_error()


def test_nothing_to_do_is_no_error():
    c, b = _cache(), _batch(n=0)
    x = torch.zeros(0, 2, 64)
    B.kv8_append(c, b, x, x)
    B.kv8_attend(c, b, _q(n=0), _q(n=0), weight=torch.zeros(2, 2, 32))


def test_codes_of_the_definition():
    """The CPU definition's rounding against torch's conversion, which is to nearest even as well, inside e4m3's range."""
    x = torch.cat([torch.randn(20000) * 64, torch.randn(20000) * 0.01, torch.tensor([0.0, -0.0, 448.0, -448.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9])])
    x = x.clamp(-448, 448)
    want = x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(K.nearest_code(x.numpy()), want)
    assert list(K.nearest_code([1e9, -math.inf, math.nan])) == [0x7E, 0xFE, 0x7F]
    assert K.power_for(np.array([448.0])) == 1.0 and K.power_for(np.array([448.0001])) == 2.0
    assert K.power_for(np.array([0.0, math.inf])) == 2.0 ** -100
