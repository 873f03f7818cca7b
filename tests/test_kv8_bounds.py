"""Arguments of the 8-bit KV cache's calls that would lead a kernel outside its tensors, or a launch past its limits: refused on the host."""
import pytest
import torch

from paper_2605_11093_amd import binding as B


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
