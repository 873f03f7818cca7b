"""The 8-bit KV cache's C interface: every declared function is exported, structs have the binding's sizes, memory that may not be
shared is refused."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_2605_11093_amd as dmi
from paper_2605_11093_amd import binding as B

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dmi_kv8.h")


def _declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return re.findall(r"\b(dmi_kv8_\w+)\s*\(", text)


def test_every_declared_function_is_exported():
    names = _declared()
    assert set(names) == {"dmi_kv8_append", "dmi_kv8_attend_workspace", "dmi_kv8_attend", "dmi_kv8_evict"}
    for name in names:
        assert getattr(B.lib(), name)
    for name in ("KV8", "KV8Batch", "kv8_append", "kv8_attend", "kv8_attend_workspace", "kv8_evict"):
        assert getattr(dmi, name) is getattr(B, name)


def test_the_header_is_plain_c(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include "dmi_kv8.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu %zu", sizeof(dmi_kv8_t), '
                   'sizeof(dmi_kv8_batch_t), sizeof(dmi_kv8_heads_t), sizeof(dmi_kv8_weight_t)); return 0; }\n')
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), str(src), "-o", exe], check=True)
    sizes = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    cache = torch.zeros(4, 16, 1, 16, dtype=torch.uint8)
    kv = B.KV8(cache, cache, torch.ones(4, 1), torch.ones(4, 1), torch.zeros(1, 4, dtype=torch.int32))
    batch = B.KV8Batch(torch.zeros(1, dtype=torch.int32), max_len=16)
    assert sizes[:2] == [len(bytes(kv._raw)), len(bytes(batch._raw))]
    assert sizes[2:] == [len(bytes(B._kv8_heads(torch.zeros(1, 1, 16), "x", 1, 1, 16))),
                         len(bytes(B._kv8_weight(torch.zeros(1, 1, 4), "x", 1, 1, 4)))]


def test_evict_refuses_weights_in_one_memory():
    def cache():
        c = torch.zeros(4, 16, 1, 16, dtype=torch.uint8)
        return B.KV8(c, c.clone(), torch.ones(4, 1), torch.ones(4, 1), torch.zeros(1, 4, dtype=torch.int32))
    w = torch.zeros(1, 1, 64)
    with pytest.raises(B.DmiError, match="to_weight is weight"):
        B.kv8_evict(cache(), B.KV8Batch(torch.zeros(1, dtype=torch.int32), max_len=64), w, cache(), w, keep=16, recent=4,
                    positions=torch.zeros(1, 1, 16, dtype=torch.int32), lens=torch.zeros(1, dtype=torch.int32))
