"""The serving loop of examples/kv8_decode.py: every step's attention against the definition in 64 bits over the cache as it stands, the
budget kept, and every step's weights observed."""
import importlib.util
import os

import pytest
import torch

import _kv8 as K

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("kv8_decode", os.path.join(ROOT, "examples", "kv8_decode.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("group,prompt,budget", [(4, 70, 48), (2, 150, 64)])
def test_serving_loop(group, prompt, budget):
    steps, heads, dim, seen_by = 12, 2, 64, []

    def check(at, cache, batch, q, out, weight, lens, spans):
        starts = [sum(spans[:i]) for i in range(len(spans))]
        rows = [(i, starts[i], spans[i], lens[i]) for i in range(len(spans))]
        cpu = K.Cpu(cache.k, cache.v, cache.k_scale, cache.v_scale, cache.block_table)
        (o, _, w), (do, _, dw) = K.attend(cpu, rows, q.cpu().double().numpy(), dim ** -0.5, group, torch.bfloat16)
        K.near(out.float().cpu().numpy(), o, do, f"out of step {at}")
        if at == 0:
            for i, n in enumerate(lens):
                K.near(weight[i, :, :n].cpu().numpy(), w[i], dw[i], f"weight of request {i}")
        seen_by.append(at)

    seen = _example().serve(requests=3, prompt=prompt, budget=budget, recent=8, slack=4, steps=steps, heads=heads, group=group, dim=dim,
                            seed=3, check=check)
    assert seen_by == list(range(steps + 1)) and seen["steps"] == seen["observed"] == steps + 1 and seen["finite"]
    assert seen["cuts"] >= 1 and max(seen["lens"]) <= budget + 4
    assert all(0.0 < kept <= 1.0 + 1e-6 for kept in seen["kept_weight"])
