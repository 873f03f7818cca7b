"""What the operators for long contexts on the 8-bit KV cache refuse, on the host, and their C interface."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_2605_11093_amd as dmi
from paper_2605_11093_amd import binding as B

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dmi_kv8_long.h")
I32 = torch.int32


def _cache(blocks=8, block=16, heads=2, dim=64, per=4, seqs=3):
    k = torch.zeros(blocks, block, heads, dim, dtype=torch.uint8)
    return B.KV8(k, k.clone(), torch.ones(blocks, heads), torch.ones(blocks, heads), torch.zeros(seqs, per, dtype=I32))


def _batch(n=3, max_len=64, **more):
    return B.KV8Batch(torch.ones(n, dtype=I32), max_len=max_len, **more)


def _refused(match, call, *a, **k):
    with pytest.raises(B.DmiError, match=match) as e:
        call(*a, **k)
    assert e.value.code == B.ERR_INVALID_ARG


def test_every_declared_function_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(dmi_kv8_\w+)\s*\(", text))
    assert names == {"dmi_kv8_append_rotated", "dmi_kv8_bound", "dmi_kv8_select_workspace", "dmi_kv8_select", "dmi_kv8_attend_blocks_workspace",
                     "dmi_kv8_attend_blocks", "dmi_kv8_attend_shared_workspace", "dmi_kv8_attend_shared"}
    for name in names:
        assert getattr(B.lib(), name) and getattr(dmi, name[4:]) is getattr(B, name[4:])
    assert dmi.KV8Rotary is B.KV8Rotary and dmi.KV8Prefix is B.KV8Prefix


def test_the_header_is_plain_c(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include "dmi_kv8_long.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu", sizeof(dmi_kv8_rotary_t), '
                   'sizeof(dmi_kv8_bounds_t), sizeof(dmi_kv8_prefix_t)); return 0; }\n')
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), str(src), "-o", exe], check=True)
    sizes = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    c = _cache()
    assert sizes == [len(B.KV8Rotary(torch.ones(8))._raw), len(B._kv8_bounds(torch.zeros(8, 2, 2, 64, dtype=torch.uint8), c)),
                     len(B.KV8Prefix(torch.zeros(2, dtype=I32), torch.zeros(1, dtype=I32), max_prefix=1)._raw)]


def _x(heads=2, n=3, dim=64, dtype=torch.bfloat16):
    return torch.zeros(n, heads, dim, dtype=dtype)


@pytest.mark.parametrize("pairs", [4, 33, 36])
def test_rotated_sizes(pairs):
    """Eight pairs at a time, and no more than a head has."""
    _refused("rotary_dim", B.kv8_append_rotated, _cache(), _batch(), _x(), _x(), B.KV8Rotary(torch.ones(pairs)))


def test_rotated_tensors():
    c, b, rot = _cache(), _batch(), B.KV8Rotary(torch.ones(32))
    _refused("different dtypes", B.kv8_append_rotated, c, b, _x(), _x(dtype=torch.float16), rot)
    _refused("different dtypes", B.kv8_append_rotated, c, b, _x(), _x(), rot, q=_x(4, dtype=torch.float32), q_out=_x(4, dtype=torch.float32))
    wide = torch.zeros(3, 6, 64, dtype=torch.bfloat16)
    _refused("q_out and q share", B.kv8_append_rotated, c, b, _x(), _x(), rot, q=wide[:, :4], q_out=wide[:, 1:5])
    _refused("q_out shares elements with key", B.kv8_append_rotated, c, b, wide[:, 4:], _x(), rot, q=_x(4), q_out=wide[:, 1:5])
    _refused("q_out shares elements with key", B.kv8_append_rotated, c, b, _x(), wide[:, :2], rot, q=_x(4), q_out=wide[:, 1:5])
    raw = B._PACK_KV8_ROTARY(rot.freq.data_ptr(), 0, 64, 2)
    rot._raw = raw
    _refused("pairs", B.kv8_append_rotated, c, b, _x(), _x(), rot)
    rot._raw = B._PACK_KV8_ROTARY(0, 0, 64, 0)
    _refused("freq_dev", B.kv8_append_rotated, c, b, _x(), _x(), rot)
    rot = B.KV8Rotary(torch.ones(32))
    with pytest.raises(ValueError, match="go together"):
        B.kv8_append_rotated(c, b, _x(), _x(), rot, q=_x(4))
    with pytest.raises(ValueError, match="positions"):
        B.kv8_append_rotated(c, b, _x(), _x(), B.KV8Rotary(torch.ones(32), positions=torch.zeros(2, dtype=I32)))
    with pytest.raises(ValueError, match="empty"):
        B.KV8Rotary(torch.ones(0))
    with pytest.raises(ValueError, match="freq"):
        B.KV8Rotary(torch.ones(8, dtype=torch.float64))


def test_queries_beside_key_and_value_in_one_tensor_are_taken():
    """In place, in the rows of a fused projection: they share memory's range and no element.  (Of no rows, so that nothing is launched.)"""
    x = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    b = B.KV8Batch(torch.ones(3, dtype=I32), max_len=0)
    B.kv8_append_rotated(_cache(), b, x[:, 4:6], x[:, 6:], B.KV8Rotary(torch.ones(32)), q=x[:, :4], q_out=x[:, :4])


def test_bounds():
    c = _cache()
    for bad in (torch.zeros(8, 2, 2, 48, dtype=torch.uint8), torch.zeros(8, 2, 2, 64), torch.zeros(7, 2, 2, 64, dtype=torch.uint8),
                torch.zeros(8, 2, 64, 2, dtype=torch.uint8).transpose(2, 3)):
        with pytest.raises(ValueError, match="bounds"):
            B.kv8_bound(c, _batch(), bad)
    odd = torch.zeros(8 * 2 * 2 * 64 + 8, dtype=torch.uint8)[8:].view(8, 2, 2, 64)
    _refused("bounds", B.kv8_bound, c, _batch(), odd)
    with pytest.raises(B.DmiError, match="bounds"):
        B._check(B.lib().dmi_kv8_bound(c._raw, _batch()._raw, None, None))


@pytest.mark.parametrize("first,recent,n", [(0, 0, 4), (3, 2, 4), (5, 1, 4), (0, 5, 4)])
def test_selections(first, recent, n):
    _refused("n_recent", B.kv8_select, _cache(), _batch(), torch.zeros(8, 2, 2, 64, dtype=torch.uint8), _x(4), torch.zeros(3, 2, n, dtype=I32), first=first,
             recent=recent)


def test_selections_tensors():
    c, b, bounds, blocks = _cache(), _batch(), torch.zeros(8, 2, 2, 64, dtype=torch.uint8), torch.zeros(3, 2, 3, dtype=I32)
    _refused("BF16 or FP16", B.kv8_select, c, b, bounds, _x(4, dtype=torch.float32), blocks)
    _refused("evenly", B.kv8_select, c, b, bounds, _x(3), blocks)
    _refused("workspace", B.kv8_select, c, b, bounds, _x(4), blocks, workspace=torch.zeros(8, dtype=torch.uint8))
    _refused("n_select", B.kv8_select, c, b, bounds, _x(4), torch.zeros(3, 2, 0, dtype=I32), workspace=torch.zeros(8, dtype=torch.uint8))
    for bad in (torch.zeros(2, 2, 3, dtype=I32), torch.zeros(3, 1, 3, dtype=I32), torch.zeros(3, 3, 2, dtype=I32).transpose(1, 2),
                torch.zeros(3, 2, 3, dtype=torch.int64)):
        with pytest.raises(ValueError, match="blocks"):
            B.kv8_select(c, b, bounds, _x(4), bad)
    assert B.kv8_select_workspace(c, b, 3) >= 3 * 2 * 4 * 8 and B.kv8_select_workspace(c, b, 4) == 0


def test_sizes_that_are_refused_have_no_workspace():
    c = _cache()
    lots = B.KV8Batch(torch.ones(1, dtype=I32), starts=torch.zeros(2, dtype=I32), total_new=1 << 30, max_new=1, max_len=1 << 24)
    assert B.kv8_select_workspace(c, lots, 8) == 0 and B.kv8_select_workspace(c, _batch(), 0) == 0
    assert B.kv8_attend_blocks_workspace(c, _batch(), 3, 8) == 0 and B.kv8_attend_blocks_workspace(c, _batch(), 4, 0) == 0
    assert B.kv8_attend_blocks_workspace(c, _batch(), 2 * 33, 8) == 0
    p = B.KV8Prefix(torch.zeros(2, dtype=I32), torch.zeros(1, dtype=I32), max_prefix=1 << 25)
    assert B.kv8_attend_shared_workspace(c, _batch(), p, 4) == 0
    p = B.KV8Prefix(torch.zeros(2, dtype=I32), torch.zeros(1, dtype=I32), max_prefix=1 << 20)
    c, b = _cache(per=1 << 16), _batch(max_len=1 << 20)
    assert B.kv8_attend_shared_workspace(c, b, p, 3) == 0 and B.kv8_attend_shared_workspace(c, b, p, 4) > 0


def test_attention_over_listed_blocks():
    c, b, blocks = _cache(), _batch(), torch.zeros(3, 2, 3, dtype=I32)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    _refused("more than 32", B.kv8_attend_blocks, c, b, blocks, _x(66), _x(66), workspace=ws)
    _refused("more than 16", B.kv8_attend_blocks, _cache(dim=256), b, blocks, _x(34, dim=256), _x(34, dim=256), workspace=ws)
    _refused("both be BF16", B.kv8_attend_blocks, c, b, blocks, _x(4), _x(4, dtype=torch.float16), workspace=ws)
    _refused("not finite", B.kv8_attend_blocks, c, b, blocks, _x(4), _x(4), scale=float("inf"), workspace=ws)
    x = torch.zeros(3, 5, 64, dtype=torch.bfloat16)
    _refused("share elements", B.kv8_attend_blocks, c, b, blocks, x[:, :4], x[:, 1:], workspace=ws)
    with pytest.raises(ValueError, match="lse"):
        B.kv8_attend_blocks(c, b, blocks, _x(4), _x(4), lse=torch.zeros(3, 3), workspace=ws)
    with pytest.raises(B.DmiError, match="blocks_dev"):
        q = B._kv8_heads(_x(4), "q", 3, 4, 64)
        B._check(B.lib().dmi_kv8_attend_blocks(c._raw, b._raw, None, 3, q, 4, 0.1, q, None, None, 0, None))


def test_attention_behind_shared_prefixes():
    c, b = _cache(), _batch()
    p = B.KV8Prefix(torch.zeros(2, dtype=I32), torch.zeros(1, dtype=I32), max_prefix=1 << 20)
    _refused("workspace", B.kv8_attend_shared, _cache(per=1 << 16), _batch(max_len=1 << 20), p, _x(4), _x(4), workspace=torch.zeros(8, dtype=torch.uint8))
    p._raw = B._PACK_KV8_PREFIX(1, 32, 0, 0)
    _refused("group_starts_dev", B.kv8_attend_shared, c, b, p, _x(4), _x(4), workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    p._raw = B._PACK_KV8_PREFIX(1 << 17, 32, 8, 8)
    _refused("n_groups", B.kv8_attend_shared, c, b, p, _x(4), _x(4), workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(ValueError, match="one entry more"):
        B.KV8Prefix(torch.zeros(1, dtype=I32), torch.zeros(1, dtype=I32), max_prefix=32)


def test_no_rows_are_no_work():
    """Calls of no requests or no new tokens return without a launch."""
    c, none = _cache(), B.KV8Batch(torch.ones(0, dtype=I32), max_len=32)
    x, bounds = _x(4, 0), torch.zeros(8, 2, 2, 64, dtype=torch.uint8)
    p = B.KV8Prefix(torch.zeros(1, dtype=I32), torch.zeros(0, dtype=I32), max_prefix=0)
    B.kv8_append_rotated(c, none, _x(2, 0), _x(2, 0), B.KV8Rotary(torch.ones(32)), q=x, q_out=x)
    B.kv8_bound(c, none, bounds)
    B.kv8_select(c, none, bounds, x, torch.zeros(0, 2, 3, dtype=I32))
    B.kv8_attend_blocks(c, none, torch.zeros(0, 2, 3, dtype=I32), x, x)
    B.kv8_attend_shared(c, none, p, x, x)
    assert C.sizeof(C.c_void_p) == 8
