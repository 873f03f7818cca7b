"""Arguments of the 8-bit KV cache's calls that would lead a kernel outside its tensors, or a launch past its limits: refused on the host."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2605_11093_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _cache(table, blocks=8, block=16, heads=2, dim=64):
    k = torch.zeros(blocks, block, heads, dim, dtype=torch.uint8)
    return B.KV8(k, k.clone(), torch.ones(blocks, heads), torch.ones(blocks, heads), table)


@pytest.mark.parametrize("table", [
    torch.zeros(1, 4, dtype=torch.int32).expand(3, -1),                     # rows that are one row
    torch.zeros(12, dtype=torch.int32).as_strided((3, 4), (2, 1)),          # rows that overlap
], ids=["expanded", "overlapping"])
def test_a_table_whose_rows_share_memory(table):
    """Its rows lie nearer to each other than they are long: no other distance stands in for the real one."""
    c, x = _cache(table), torch.zeros(3, 2, 64)
    with pytest.raises(B.DmiError, match="block_table_stride") as e:
        B.kv8_append(c, B.KV8Batch(torch.ones(3, dtype=torch.int32), max_len=32), x, x)
    assert e.value.code == B.ERR_INVALID_ARG


def test_a_table_of_one_row_may_have_any_stride():
    c = _cache(torch.zeros(4, dtype=torch.int32).as_strided((1, 4), (0, 1)))
    x = torch.zeros(0, 2, 64)
    B.kv8_append(c, B.KV8Batch(torch.ones(0, dtype=torch.int32), max_len=32), x, x)


_WORKSPACE = """
import sys
from paper_2605_11093_amd import binding as B
heads, dim, q_heads, reqs, total, new, length = map(int, sys.argv[1:])
cache = B._PACK_KV8(0, 0, 0, 0, 0, 0, 0, 0, 0, 16, heads, dim, 1, 1, 1, 0, 1)
print(B.lib().dmi_kv8_attend_workspace(cache, B._PACK_KV8_BATCH(reqs, total, new, length, 0, 0, 0), q_heads, 1))
"""


def _workspace(*numbers):
    p = subprocess.run([sys.executable, "-c", _WORKSPACE, *map(str, numbers)], capture_output=True, text=True, cwd=ROOT)
    assert p.returncode == 0, f"ended by {p.returncode}: {p.stderr}"
    return int(p.stdout)


@pytest.mark.parametrize("numbers", [
    (1 << 31, 256, 1 << 31, 1, 32, 32, 100),        # heads whose tiles of query rows are more than 32 bits count
    (2048, 64, 2048, 1, 1, 1, 100), (2, 512, 4, 1, 1, 1, 100), (2, 0, 4, 1, 1, 1, 100), (2, 64, 3, 1, 1, 1, 100),
    (1, 64, 1 << 17, 1, 1, 1, 100), (2, 64, 4, 1 << 17, 1 << 17, 1, 100), (2, 64, 4, 1, 1, 1, 1 << 25),
    (2, 64, 4, 1, 1 << 31, 1, 100), (2, 64, 4, 1, 1 << 20, 1 << 25, 100)],
    ids=["tiles", "heads", "dim", "no dim", "uneven", "q heads", "requests", "length", "rows", "new"])
def test_workspace_of_sizes_that_attend_refuses(numbers):
    """In a process of its own: a division by zero would end it."""
    assert _workspace(*numbers) == 0


def test_workspace_of_sizes_that_attend_takes():
    assert _workspace(8, 128, 32, 16, 16, 1, 8192) >= 16 * 32 * 8192 * 4


@pytest.mark.parametrize("numbers", [
    (1, 64, 2, 1, 1 << 30, 16, 1 << 24),            # scores of more bytes than 64 bits count
    (1024, 64, 1 << 15, 1, 1 << 30, 1, 1 << 24),
    (1, 64, 65536, 1, 1 << 30, 1 << 24, 100),       # query rows of one request past 32 bits
], ids=["scores", "heads", "rows"])
def test_more_query_rows_than_31_bits_count(numbers):
    """Sizes in bytes would wrap, and rows of a request: refused by the workspace's function and by the call."""
    heads, dim, q_heads, reqs, total, new, length = numbers
    assert _workspace(*numbers) == 0
    blocks = -(-length // 16)
    word = torch.zeros(4, dtype=torch.int32)
    code = (16 - word.data_ptr() % 16) % 16 + word.data_ptr()
    # (pointers are only looked at: it is refused before anything is launched)
    cache = B._PACK_KV8(code, code, code, code, 16 * heads * 64, heads * 64, 64, heads, 1, 16, heads, dim, 1, 1, blocks, code, blocks)
    batch = B._PACK_KV8_BATCH(reqs, total, new, length, code, code, 0)
    rows = B._PACK_KV8_HEADS(code, B.DT_BF16, q_heads * dim, dim)
    weight = B._PACK_KV8_WEIGHT(code, heads * length, length)
    assert B.lib().dmi_kv8_attend(cache, batch, rows, q_heads, 1.0, rows, None, weight, None, 0.0, 256, 1 << 62, None) == B.ERR_INVALID_ARG
    assert b"total_new" in B.lib().dmi_last_error()


def _pointer():
    word = torch.zeros(64, dtype=torch.int32)
    return (256 - word.data_ptr() % 256) % 256 + word.data_ptr()


@pytest.mark.parametrize("group,new", [(1, 1), (1, 64)], ids=["few", "many"])
def test_attend_past_the_workgroups_of_a_launch(group, new):
    """Weights of 2^24 positions of 1024 heads: more workgroups than a launch has, found before the first of its launches."""
    heads, length, at = 1024, 1 << 24, _pointer()
    cache = B._PACK_KV8(at, at, at, at, 16 * heads * 64, heads * 64, 64, heads, 1, 16, heads, 64, 1, 1, length // 16, at, length // 16)
    batch = B._PACK_KV8_BATCH(1, new, new, length, at, at, 0)
    q, out = (B._PACK_KV8_HEADS(at + x, B.DT_BF16, heads * 64, 64) for x in (0, 1 << 40))
    weight = B._PACK_KV8_WEIGHT(at, heads * length, length)
    assert B.lib().dmi_kv8_attend(cache, batch, q, heads * group, 1.0, out, None, weight, None, 0.0, 256, 1 << 62, None) == B.ERR_INVALID_ARG
    assert b"launch" in B.lib().dmi_last_error()


def test_evict_past_the_workgroups_of_a_launch():
    heads, keep, at = 1024, 1 << 24, _pointer()
    cache = B._PACK_KV8(at, at, at, at, 16 * heads * 64, heads * 64, 64, heads, 1, 16, heads, 64, 1, 64, keep // 16, at, keep // 16)
    batch = B._PACK_KV8_BATCH(64, 0, 0, keep, at, 0, 0)
    w, to_w = (B._PACK_KV8_WEIGHT(x, heads * keep, keep) for x in (at, at + 64))
    assert B.lib().dmi_kv8_evict(cache, batch, w, cache, to_w, keep, 1, at, at + 4096, None) == B.ERR_INVALID_ARG
    assert b"launch" in B.lib().dmi_last_error()


def test_append_past_the_workgroups_of_a_launch():
    heads, new, at = 1024, 1 << 24, _pointer()
    cache = B._PACK_KV8(at, at, at, at, 16 * heads * 64, heads * 64, 64, heads, 1, 16, heads, 64, 1, 1, new // 16, at, new // 16)
    batch = B._PACK_KV8_BATCH(1, new, new, new, at, at, 0)
    x = B._PACK_KV8_HEADS(at, B.DT_BF16, heads * 64, 64)
    assert B.lib().dmi_kv8_append(cache, batch, x, x, None) == B.ERR_INVALID_ARG
    assert b"launch" in B.lib().dmi_last_error()


@pytest.mark.parametrize("rows", [1, 40], ids=["few", "many"])
def test_weights_with_outputs_in_the_queries_memory(rows):
    """Weights of many query rows are computed behind the outputs, out of the queries: both in one memory are refused, whatever the rows;
    slices of one tensor that share no element are not."""
    k = torch.zeros(8, 16, 2, 64, dtype=torch.uint8)
    c = B.KV8(k, k.clone(), torch.ones(8, 2), torch.ones(8, 2), torch.zeros(1, 4, dtype=torch.int32))
    batch = B.KV8Batch(torch.ones(1, dtype=torch.int32), max_len=64, starts=torch.zeros(2, dtype=torch.int32), total_new=rows, max_new=rows)
    w, both = torch.zeros(1, 2, 64), torch.zeros(rows, 8, 144, dtype=torch.bfloat16)

    def call(q, out, weight):
        with pytest.raises(B.DmiError) as e:    # (refused, or no device to launch on)
            B.kv8_attend(c, batch, q, out, weight=weight)
        return "same memory" in str(e.value)
    q = both[:, :4, :64]
    assert call(q, q, w) and not call(q, q, None)
    assert call(q, both[:, 2:6, :64], w) and call(q, both[:, 3:7, :64], w)
    assert call(both[:, :, :64][:, ::2], both[:, :4, 48:112], w) and call(both[:, 1:5, :64], both[:, :4, :64], w)
    assert not call(q, both[:, 4:, :64], w) and not call(q, both[:, :4, 80:], w) and not call(both[:, ::2, :64], both[:, 1::2, :64], w)
    assert not call(q, torch.zeros(rows, 4, 64, dtype=torch.bfloat16), w)
    if rows > 1:
        wide = torch.zeros(rows + 1, 4, 64, dtype=torch.bfloat16)
        assert call(wide[1:], wide[:-1], w)


def test_more_tokens_than_tiles_are_counted():
    """Tiles of 32 tokens of all contexts are added up in 31 bits: lengths that a sum would wrap for are refused by their bound."""
    reqs, length, at = 65535, 1 << 24, _pointer()
    assert _workspace(1, 64, 1, reqs, reqs, 1, length) == 0 and _workspace(1, 64, 1, 1024, 1024, 1, length) > 0
    cache = B._PACK_KV8(at, at, at, at, 16 * 64, 64, 64, 1, 1, 16, 1, 64, 1, reqs, length // 16, at, length // 16)
    batch = B._PACK_KV8_BATCH(reqs, reqs, 1, length, at, 0, 0)
    q, out = (B._PACK_KV8_HEADS(at + x, B.DT_BF16, 64, 64) for x in (0, 1 << 40))
    assert B.lib().dmi_kv8_attend(cache, batch, q, 1, 1.0, out, None, None, None, 0.0, 256, 1 << 62, None) == B.ERR_INVALID_ARG
    assert b"2^35" in B.lib().dmi_last_error()


def test_new_lengths_inside_the_lengths():
    """to_lens_dev anywhere in lens_dev's memory: the move would take other requests' new lengths for their lengths."""
    both, w = torch.ones(5, dtype=torch.int32), torch.zeros(2, 3, 2, 64)
    c, to = (_cache(torch.zeros(3, 4, dtype=torch.int32)) for _ in range(2))
    positions = torch.zeros(3, 2, 16, dtype=torch.int32)
    for lens, new in ((both[:3], both[2:]), (both[1:4], both[:3]), (both[:3], both[:3])):
        with pytest.raises(B.DmiError, match="lens_dev") as e:
            B.kv8_evict(c, B.KV8Batch(lens, max_len=64), w[0], to, w[1], keep=16, recent=4, positions=positions, lens=new)
        assert e.value.code == B.ERR_INVALID_ARG


def _select(reqs, total, length, *, heads=8, group=4, n_select=64, call=True):
    """dmi_kv8_select's status (or its workspace) for `total` new tokens over up to `length`, by addresses that nothing looks at."""
    at = _pointer()
    cache = B._PACK_KV8(at, at, at, at, 16 * heads * 128, heads * 128, 128, heads, 1, 16, heads, 128, 1, reqs, length // 16, at, length // 16)
    batch = B._PACK_KV8_BATCH(reqs, total, total, length, at, at, 0)
    if not call:
        return B.lib().dmi_kv8_select_workspace(cache, batch, n_select)
    q = B._PACK_KV8_HEADS(at, B.DT_BF16, heads * group * 128, 128)
    return B.lib().dmi_kv8_select(cache, batch, B._PACK_KV8_BOUNDS(at, heads * 256, 256), q, heads * group, n_select, 1, 2, at, 256, 1 << 62, None)


NO_DEVICE = pytest.mark.skipif(torch.cuda.is_available(), reason="launches by addresses that are none")


@NO_DEVICE
@pytest.mark.parametrize("reqs,total,length,group", [
    (1, 32768, 131072, 4),              # a part of a long prompt, one launch
    (1, 1 << 19, 131072, 4), (64, 1 << 20, 16 * 3000, 4), (4, 1 << 21, 16 * 3000, 2), (1, 4000000, 16 * 1000, 8)])
def test_select_of_no_more_workgroups_than_a_launch_has(reqs, total, length, group):
    """What a path launches is what it is refused for, not what another one would: only a device is missing."""
    assert _select(reqs, total, length, call=False) > 0
    assert _select(reqs, total, length, group=group) == B.ERR_HIP, B.lib().dmi_last_error()


@pytest.mark.parametrize("reqs,total,length", [(1, 1 << 24, 131072), (4, 1 << 23, 16 * 3000), (1, 1 << 17, 16 * 400000)], ids=["one launch", "several", "two"])
def test_select_past_the_workgroups_of_a_launch(reqs, total, length):
    assert _select(reqs, total, length) == B.ERR_INVALID_ARG and b"launch" in B.lib().dmi_last_error()


@pytest.mark.parametrize("total,length", [(128, 8192), (3, 16 * 900), (32768, 131072), (760, 50000)])
def test_workspace_of_a_selection_in_one_launch(total, length):
    """Its scores lie in LDS: what it keeps in memory is a word of 8 bytes for each, and no more."""
    assert total * 8 * (length // 16) * 8 <= _select(1, total, length, call=False) <= total * 8 * (length // 16) * 8 + 256


@pytest.mark.parametrize("total,length", [(4, 16 * 7500), (3, 16 * 9000)])
def test_workspace_of_a_selection_in_two_launches(total, length):
    """Scores with what they may be off, and a word for each."""
    assert _select(1, total, length, call=False) >= total * 8 * (length // 16) * 16


def _attend(call, reqs, heads, total, new, length, *more, dim=64, starts=True):
    """The status of an attention for long contexts, by addresses that nothing looks at."""
    at = _pointer()
    cache = B._PACK_KV8(at, at, at, at, 16 * heads * dim, heads * dim, dim, heads, 1, 16, heads, dim, 1, reqs, -(-length // 16), at, -(-length // 16))
    batch = B._PACK_KV8_BATCH(reqs, total, new, length, at, at if starts else 0, 0)
    q, out = (B._PACK_KV8_HEADS(at + x, B.DT_BF16, heads * dim, dim) for x in (0, 1 << 40))
    if call == "blocks":
        return B.lib().dmi_kv8_attend_blocks(cache, batch, at, more[0], q, heads, 1.0, out, None, 256, 1 << 62, None)
    prefix = B._PACK_KV8_PREFIX(1, more[0], at, at)
    return B.lib().dmi_kv8_attend_shared(cache, batch, prefix, q, heads, 1.0, out, None, 256, 1 << 62, None)


@pytest.mark.parametrize("reqs,heads,total,new,length", [(4096, 64, 4096, 1, 500000), (65535, 256, 65535, 1, 20000), (40000, 256, 1 << 22, 256, 20000)],
                         ids=["single tokens", "more of them", "prompts"])
def test_attend_shared_past_the_workgroups_of_a_launch(reqs, heads, total, new, length):
    """What is behind prefixes takes more workgroups than a launch has, prefixes do not: found before the prefixes' launch."""
    assert _attend("shared", reqs, heads, total, new, length, 64, starts=new > 1) == B.ERR_INVALID_ARG and b"launch" in B.lib().dmi_last_error()


@NO_DEVICE
@pytest.mark.parametrize("total,heads,n_select", [(1 << 20, 8, 8), (1 << 20, 16, 64), (1 << 22, 8, 8)])
def test_attend_blocks_of_no_more_workgroups_than_a_launch_has(total, heads, n_select):
    """A wavefront for each of many lists is a workgroup of 64 threads: only a device is missing."""
    assert _attend("blocks", 32, heads, total, total, 65536, n_select) == B.ERR_HIP, B.lib().dmi_last_error()


def test_attend_blocks_past_the_workgroups_of_a_launch():
    assert _attend("blocks", 32, 64, 1 << 21, 1 << 21, 65536, 8) == B.ERR_INVALID_ARG and b"launch" in B.lib().dmi_last_error()
