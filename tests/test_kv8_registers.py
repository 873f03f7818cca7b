"""Kernels of the 8-bit KV cache leave registers free: one that fills all 512 parks values in accumulator registers, also where some lanes
are switched off, and lanes that were off read back something else."""
import subprocess

import test_kernel_resources as R


def test_no_kernel_fills_the_registers():
    data = open(R.SO, "rb").read()
    seen = 0
    for elf in R._code_objects(data):
        for kernel in R._kernels(elf):
            name = subprocess.run(["c++filt", kernel[".name"]], capture_output=True, text=True).stdout
            if "dmi::kv8::" not in name:
                continue
            seen += 1
            assert kernel[".vgpr_count"] < 512 and kernel[".vgpr_spill_count"] == 0, name
    assert seen >= 30
