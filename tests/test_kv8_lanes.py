"""Kernels of the 8-bit KV cache as built: none parks a value where some of the lanes that need it are switched off.  A block that several
paths lead to begins with bringing the other lanes back; the compiler, out of vector registers, once put a copy into an accumulator
register in front of that, and the lanes that were off read back what the register had held before."""
import os
import re
import shutil
import subprocess

import pytest

import test_kernel_resources as R

OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"


def parked(text):
    """Copies into accumulator registers or to scratch memory at the head of a block, in front of its restoring of exec: (label, line)."""
    found = []
    for block in re.split(r"^(?=<?[.\w]+>?:\s*$)", text, flags=re.M):
        lines = [x.split("//")[0].strip() for x in block.split("\n")]
        head = []
        for line in lines[1:]:
            op = line.split()[0] if line else ""
            if op in ("s_or_b64", "s_mov_b64") and line.split()[1] == "exec,":
                found += [(lines[0], x) for x in head]
                break
            if op.startswith(("s_cbranch", "s_branch", "s_setpc", "s_endpgm", "s_barrier")) or "saveexec" in op:
                break
            if op.startswith(("v_accvgpr_write", "v_accvgpr_mov", "scratch_store")):
                head.append(line)
    return found


def labelled(part):
    """A kernel's listing with a label in front of every instruction that a branch leads to."""
    base = int(part[:part.index(" ")], 16)
    targets = {base + int(x, 16) for x in re.findall(r"s_c?branch.*<\S+\+0x([0-9a-f]+)>", part)}
    out = []
    for line in part.split("\n")[1:]:
        at = re.search(r"// ([0-9A-F]{12}):", line)
        if at and int(at.group(1), 16) in targets:
            out.append(f"<L{at.group(1)}>:")
        out.append(line)
    return "\n".join(out), len(targets)


def test_the_case_that_was_seen():
    seen = "<L7>:\n\tv_accvgpr_write_b32 a160, v132 // 0001: 2\n\ts_or_b64 exec, exec, s[4:5]\n\tv_add_f32 v1, v2, v3\n"
    assert parked(seen) == [("<L7>:", "v_accvgpr_write_b32 a160, v132")]
    assert not parked(seen.replace("<L7>:\n", "<L7>:\n\ts_or_b64 exec, exec, s[4:5]\n", 1).replace("v_add_f32", "s_endpgm\n", 1))
    assert not parked("<L8>:\n\tv_accvgpr_write_b32 a1, v2\n\ts_cbranch_vccz L9\n\ts_or_b64 exec, exec, s[0:1]\n")


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler here")
def test_nothing_is_parked_where_lanes_are_off(tmp_path):
    if not os.path.exists(R.SO):
        pytest.skip("the library has not been built")
    kernels = 0
    for i, elf in enumerate(R._code_objects(open(R.SO, "rb").read())):
        if not any("3kv8" in k[".name"] for k in R._kernels(elf)):
            continue
        path = tmp_path / f"{i}.elf"
        path.write_bytes(elf)
        text = subprocess.run([OBJDUMP, "-d", str(path)], capture_output=True, text=True, check=True).stdout
        for part in re.split(r"^(?=[0-9a-f]+ <_Z)", text, flags=re.M)[1:]:
            name = part[part.index("<") + 1:part.index(">")]
            if "3kv8" not in name:
                continue
            kernels += 1
            listing, blocks = labelled(part)
            assert blocks > 3 and listing.count("\n<L") + listing.startswith("<L") == blocks, name      # (blocks were told apart)
            assert not parked(listing), (name, parked(listing)[:3])
    assert kernels >= 30
