"""A serving loop over the 8-bit KV cache: prompts are appended and attended to, requests that outgrow their budget keep the tokens
that received the most attention, and single tokens are decoded; the weights that decide it are observed on the way.

One layer of random projections stands in for a model.  Per step: append -> attend (with weights) -> now and then evict, all on
one stream; the weight rows go through a ring like any other activation.  Only a cut is waited for: the host hands out blocks, so
it has to know the new lengths.

    python examples/kv8_decode.py [--requests 8] [--prompt 900] [--budget 512] [--steps 64] ...
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_11093_amd import binding as B                      # noqa: E402

POINT = 7                                                           # of the observed weights


class Pool:
    """Blocks of a cache in 8 bits, and which of them are free."""

    def __init__(self, n_blocks, block, heads, dim, device):
        self.codes = torch.zeros(2, n_blocks, block, heads, dim, dtype=torch.uint8, device=device)
        self.scales = torch.ones(2, n_blocks, heads, device=device)
        self.block, self.free = block, list(range(n_blocks))

    def grow(self, blocks, tokens):
        """A request's list of blocks made long enough for `tokens`."""
        while len(blocks) * self.block < tokens:
            blocks.append(self.free.pop())

    def view(self, lists, columns):
        """The cache as these lists of blocks see it."""
        table = torch.tensor([b + [-1] * (columns - len(b)) for b in lists], dtype=torch.int32).to(self.codes.device)
        return B.KV8(self.codes[0], self.codes[1], self.scales[0], self.scales[1], table)


class Layer:
    def __init__(self, heads, group, dim, device, generator):
        width = heads * group * dim
        self.heads, self.group, self.dim = heads, group, dim

        def made(n, gain):
            return (torch.randn(width, n, generator=generator) * gain * width ** -0.5).to(device, torch.bfloat16)

        self.q, self.k, self.v, self.o = made(width, 2.0), made(heads * dim, 2.0), made(heads * dim, 1.0), made(width, 1.0)

    def project(self, x):
        n = x.shape[0]
        return ((x @ self.q).view(n, -1, self.dim), (x @ self.k).view(n, -1, self.dim), (x @ self.v).view(n, -1, self.dim))

    def finish(self, x, out):
        y = x.float() + (out.reshape(x.shape) @ self.o).float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def serve(requests=8, prompt=900, budget=512, recent=64, slack=32, steps=64, heads=8, group=4, dim=128, block=16, decay=0.95,
          device="cuda:0", seed=0, check=None):
    """Returns what happened; `check` sees every step's cache, batch, rows and weights."""
    g = torch.Generator().manual_seed(seed)
    layer = Layer(heads, group, dim, device, g)
    stream = torch.cuda.current_stream(device).cuda_stream
    lens = torch.randint(1, prompt + 1, (requests,), generator=g).tolist()
    longest = max(max(lens), budget) + slack + 1
    columns = -(-longest // block)
    pool = Pool(2 * requests * columns, block, heads, dim, device)
    lists = [[] for _ in range(requests)]
    weight = torch.zeros(requests, heads, columns * block, device=device)
    spare, positions = torch.zeros_like(weight), torch.empty(requests, heads, budget, dtype=torch.int32, device=device)
    new_lens = torch.empty(requests, dtype=torch.int32, device=device)
    seen = {"steps": 0, "cuts": 0, "kept_weight": [], "observed": 0, "tokens": 0}

    def step(x, spans, ring, at):
        nonlocal weight, spare, lists
        q, k, v = layer.project(x)
        out = torch.empty_like(q)
        for i, n in enumerate(lens):
            pool.grow(lists[i], n)
        cache = pool.view(lists, columns)
        starts = torch.tensor([0] + spans, dtype=torch.int32).cumsum(0).to(device, torch.int32)
        batch = B.KV8Batch(torch.tensor(lens, dtype=torch.int32).to(device), starts=starts, total_new=sum(spans), max_new=max(spans),
                           max_len=max(lens))
        B.kv8_append(cache, batch, k, v, stream=stream)
        B.kv8_attend(cache, batch, q, out, weight=weight, prior=weight if at else None, decay=decay, stream=stream)
        if check is not None:
            check(at, cache, batch, q, out, weight, lens, spans)
        # every head's weights of every request, one record; what lies behind a request's length is left from longer times
        ring.observe_tensor(POINT, weight.view(requests * heads, -1), [(i, 0, i * heads, heads, 1) for i in range(requests)],
                            step_id=at, stream=stream, summary_mask=1)
        seen["observed"] += taken(ring, 0)
        seen["steps"] += 1
        seen["tokens"] += sum(spans)
        if max(lens) > budget + slack:
            cut = [[] for _ in range(requests)]
            for i, n in enumerate(lens):
                pool.grow(cut[i], min(n, budget))
            to = pool.view(cut, columns)
            B.kv8_evict(cache, batch, weight, to, spare, keep=budget, recent=recent, positions=positions, lens=new_lens, stream=stream)
            before, after = (sum(float(w[i, :, :n].sum()) for i, n in enumerate(ns))
                             for w, ns in ((weight, lens), (spare, [min(n, budget) for n in lens])))
            seen["kept_weight"].append(after / before)
            for blocks in lists:
                pool.free += blocks
            lists, weight, spare = cut, spare, weight
            lens[:] = new_lens.tolist()
            seen["cuts"] += 1
        return layer.finish(x, out)

    with B.Ring(64 << 20, 64 << 20) as ring:
        x = torch.randn(sum(lens), heads * group * dim, generator=g).to(device, torch.bfloat16)
        spans = list(lens)
        last = torch.tensor(spans).cumsum(0).to(device) - 1
        x = step(x, spans, ring, 0)[last]
        for at in range(1, steps + 1):
            for i in range(requests):
                lens[i] += 1
            x = step(x, [1] * requests, ring, at)
        seen["observed"] += taken(ring, B.DRAIN_FLUSH)
    seen["lens"], seen["finite"] = list(lens), bool(torch.isfinite(x.float()).all())
    seen["bits"] = 8 * (1 + 4 / (block * dim))                      # of a cached number, scales included
    return seen


def taken(ring, flags):
    """How many records have reached the host; they are given back to the ring."""
    ring.drain(flags)
    views = ring.poll_host()
    if views:
        ring.release_host(views[-1].seq)
    return len(views)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("requests", 8), ("prompt", 900), ("budget", 512), ("recent", 64), ("steps", 64), ("heads", 8), ("group", 4),
                        ("dim", 128), ("block", 16)):
        p.add_argument(f"--{name}", type=int, default=value)
    seen = serve(**vars(p.parse_args()))
    print(f"{seen['tokens']} tokens in {seen['steps']} steps, {seen['cuts']} cuts that kept "
          f"{', '.join(f'{k:.2f}' for k in seen['kept_weight']) or 'nothing'} of the weight, {seen['observed']} records, "
          f"{seen['bits']:.2f} bits a cached number, lengths now {seen['lens']}")
    if not seen["finite"]:
        raise SystemExit("the outputs are not finite")


if __name__ == "__main__":
    main()
