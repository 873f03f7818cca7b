"""The sources of the operators on the 8-bit KV cache, as one program: a type of dmi::kv8 has one definition."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_11093_amd", "csrc")


def test_a_type_is_defined_once():
    """Two definitions with different members under one name are undefined behaviour, whether or not a linker ever sees both."""
    where = {}
    for path in sorted(glob.glob(os.path.join(CSRC, "dmi_kv8*"))):
        # (at the start of a line: those inside of functions are their own)
        for name in re.findall(r"^(?:template\s*<(?!>)[^>]*>\s*)?struct\s+(\w+)\s*\{", open(path).read(), flags=re.M):
            where.setdefault(name, []).append(os.path.basename(path))
    assert {"Cache", "Bf16", "Fp16", "Eight", "Request", "TokensPlan"} <= set(where)
    assert not {name: files for name, files in where.items() if len(files) > 1}
