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


def test_rows_handed_over_in_lds_wait():
    """parts_kernel hands rows from lanes to other lanes of their wavefront through LDS.  Whoever reads what other lanes have written, or
    writes where they read, does so behind a point that the compiler moves no access over."""
    text = open(os.path.join(CSRC, "dmi_kv8_parts.hip")).read()
    text = text[text.index("auto in_row ="):text.index("join_parts_kernel")]
    text = text[text.index(";") + 1:]
    seen = ""
    for m in re.finditer(r"(reinterpret_cast<(const )?\w+ \*>\(in_row\()|(\blds_barrier\(\))|(\blds_handover\(\))", text):
        seen += "S" if not m.group(1) else "R" if m.group(2) else "W"
    runs = re.sub(r"(.)\1+", r"\1", seen)
    assert runs.count("W") == runs.count("R") == 3, runs
    assert "WR" not in runs and "RW" not in runs, runs
    assert runs.endswith("WSRS")                # (the last two are in a loop)
