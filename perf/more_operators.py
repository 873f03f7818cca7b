"""The operators for long contexts on a paged KV cache held in 8 bits, as cases that can be timed and compared.

Five kinds of case, one per operator:

  rotate   new tokens' K rotated by their positions and written into the cache with V (e4m3 codes, a power of two as scale per
           block of tokens and head), their queries rotated on the way
  bound    the least and the largest K of every block that new tokens reach, per head and element, as codes of the cache
  select   for each new token and head of the cache, the blocks whose bounds leave room for the largest scores, among them the
           first and the newest ones
  blocks   attention of each new token over the blocks that are listed for it and each head
  shared   causal attention of requests whose groups share their first tokens: a group's whole shared blocks are read once

A request has a row in the block table; its length counts the tokens of the call.  Codes come out as e4m3 numbers, next to the
scales that multiply them.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
LARGEST = 448.0                 # the largest e4m3 number


def _case(name, kind, dtype, reqs, lens, new, **more):
    """lens: tokens in the cache before the call's own (behind the shared ones, where there are), new: the call's own, both as
    (lowest, highest) per request."""
    return {"name": name, "kind": kind, "dtype": dtype, "reqs": reqs, "seqs": reqs, "len_lo": lens[0], "len_hi": lens[1],
            "new_lo": new[0], "new_hi": new[1], "heads": 8, "group": 4, "dim": 128, "block": 16, "order": "slots", "fused": False,
            "rotary": 0, "pairs": False, "moved": 0, "select": 0, "first": 0, "recent": 0, "groups": 0, "prefix_lo": 0, "prefix_hi": 0,
            **more}


def listed():
    return [
        # one decode step's tokens of four short requests: nothing but latency
        _case("rotate_tokens_few", "rotate", "bf16", 4, (32, 64), (1, 1), rotary=128, fused=True),
        # ragged prompts of an 8B-shaped model, as in the prefill configuration, out of a fused projection
        _case("rotate_prompts", "rotate", "bf16", 32, (0, 0), (128, 2048), rotary=128, fused=True),
        # later parts of prompts whose caches have been cut, so that positions run ahead of places; a part of each head, neighbours in
        # pairs, in single precision, heads of odd size
        _case("rotate_parts_odd", "rotate", "fp32", 16, (1, 1000), (1, 500), dim=80, block=32, heads=4, rotary=48, pairs=True, moved=100000),
        # behind a decode step of the paged configuration's 128 requests
        _case("bound_tokens", "bound", "bf16", 128, (511, 8191), (1, 1)),
        # behind the prompts above
        _case("bound_prompts", "bound", "bf16", 32, (0, 0), (128, 2048)),
        # a decode step of the paged configuration's 128 requests, of which each reads 1024 tokens
        _case("select_tokens", "select", "bf16", 128, (511, 8191), (1, 1), select=64, first=1, recent=4),
        # four requests with long contexts, heads of a small model
        _case("select_long", "select", "fp16", 4, (60000, 120000), (1, 1), select=128, first=4, recent=16, heads=4, dim=64),
        # the attention behind the selections of the 128
        _case("blocks_tokens", "blocks", "bf16", 128, (511, 8191), (1, 1), select=64, first=1, recent=4),
        # three tokens a request to verify over long contexts, cache laid out head by head, larger blocks
        _case("blocks_verify", "blocks", "fp16", 8, (8000, 30000), (3, 3), select=32, first=1, recent=2, heads=4, dim=64, block=64, order="heads"),
        # a decode step of 64 requests behind one long prompt of 8192 tokens
        _case("shared_tokens", "shared", "bf16", 64, (15, 1023), (1, 1), groups=1, prefix_lo=8192, prefix_hi=8192),
        # three tokens a request to verify, four short prompts that a few requests each share, which end inside of blocks
        _case("shared_groups", "shared", "fp16", 24, (20, 400), (3, 3), groups=4, prefix_lo=500, prefix_hi=2000, heads=4, dim=64),
        # ragged prompts behind one prompt that all begin with: the most arithmetic
        _case("shared_prompts", "shared", "bf16", 32, (0, 0), (32, 512), groups=1, prefix_lo=4000, prefix_hi=4000, fused=True),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "bound", "select", "select", "blocks", "blocks", "shared", "shared", "shared"])
    heads, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 4, 4, 7, 8])
    hi = _log(rng, 4, 16384)
    c = _case("", kind, rng.choice(["bf16", "bf16", "fp16"]), _log(rng, 1, 128), (rng.randint(0, hi), hi), (0, 0), heads=heads,
              group=group, dim=rng.choice([64, 80, 96, 128, 128, 256]), block=rng.choice([16, 16, 32, 64]),
              order=rng.choice(["slots", "slots", "heads"]), fused=rng.random() < 0.3)
    new = rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 8, 2048 if kind in ("rotate", "bound", "shared") else 256)])
    c["new_lo"], c["new_hi"] = (new, new) if new < 9 else (rng.randint(1, new), new)
    if new > 8 and rng.random() < 0.5:
        c["len_lo"] = c["len_hi"] = 0
    if kind == "rotate":
        c["dtype"] = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        c["rotary"] = c["dim"] if rng.random() < 0.6 else 16 * rng.randint(1, c["dim"] // 16)
        c["pairs"], c["moved"] = rng.random() < 0.4, rng.choice([0, 0, _log(rng, 10, 1000000)])
    elif kind in ("select", "blocks"):
        if rng.random() < 0.2:
            c["len_hi"] = _log(rng, 16384, 131072)
            c["reqs"] = min(c["reqs"], 4)
        c["len_hi"] = max(c["len_hi"], _log(rng, 256, 16384))
        c["first"], c["recent"] = rng.randint(0, 4), rng.randint(1, 8)
        c["select"] = c["first"] + c["recent"] + _log(rng, 1, 120)
    elif kind == "shared":
        c["prefix_hi"] = _log(rng, 16, 8192)
        c["prefix_lo"] = rng.randint(1, c["prefix_hi"])
        c["groups"] = min(c["reqs"], rng.choice([1, 1, rng.randint(2, 8)]))
        c["len_hi"] = _log(rng, 4, 2048)
        c["len_lo"] = rng.randint(0, c["len_hi"])
    del c["name"]
    # no dearer than the listed ones
    while True:
        w, n = work(c), _lengths(c)
        total, longest = sum(m for m, _ in n), max(t for _, t in n)
        pad, scores = len(n) * longest * c["heads"], 0
        if kind == "shared":
            scores = pad * c["group"] * max(m for m, _ in n)
        elif kind == "blocks":
            scores = total * c["heads"] * c["select"] * c["block"] * c["dim"]
        elif kind == "select":
            scores = 4 * total * c["heads"] * c["group"] * longest // c["block"] + len(n) * longest // c["block"] * c["dim"] * c["heads"]
        if w["bytes"] <= 800e6 and w["flops"] <= 2e11 and pad * c["dim"] <= 1 << 30 and scores <= 1 << 30 and total * c["heads"] * c["group"] * c["dim"] <= 1 << 28:
            c["seqs"] = c["reqs"] if rng.random() < 0.6 else c["reqs"] + rng.randint(1, 8)
            return c
        for k in ("reqs", "len_hi", "new_hi", "heads", "group"):
            if c[k] > 1 and rng.random() < 0.5:
                c[k] = c[k] // 2
        c["len_lo"], c["new_lo"], c["groups"] = min(c["len_lo"], c["len_hi"]), min(c["new_lo"], c["new_hi"]), min(c["groups"], c["reqs"])


# ------------------------------------------------------------------ what a case asks for
def _prefixes(c):
    """(first request behind it, shared tokens) of every group: the case alone fixes them."""
    r = random.Random("%(groups)d %(reqs)d %(prefix_lo)d %(prefix_hi)d" % c)
    ends = sorted(r.sample(range(1, c["reqs"]), c["groups"] - 1)) + [c["reqs"]] if c["groups"] else []
    return [(end, r.randint(c["prefix_lo"], c["prefix_hi"])) for end in ends]


def _lengths(c):
    """(new tokens, tokens with them) per request: the case alone fixes them, so every seed asks for the same work."""
    r = random.Random("%(kind)s %(reqs)d %(len_lo)d %(len_hi)d %(new_lo)d %(new_hi)d" % c)
    out, groups = [], _prefixes(c)
    for i in range(c["reqs"]):
        new = r.randint(c["new_lo"], c["new_hi"])
        before = next((p for end, p in groups if i < end), 0)
        out.append((new, before + r.randint(c["len_lo"], c["len_hi"]) + new))
    return out


def _most(c):
    """The longest context that a request's row of the block table has room for."""
    return c["prefix_hi"] + c["len_hi"] + max(1, c["new_hi"])


def work(case):
    c, n = case, _lengths(case)
    new, tokens = sum(m for m, _ in n), sum(t for _, t in n)
    heads, group, d, size, bs = c["heads"], c["group"], c["dim"], SIZE[c["dtype"]], c["block"]
    rows = new * heads * group
    touched = sum(-(-t // bs) - (t - m) // bs for m, t in n)
    if c["kind"] == "rotate":
        moved = 2 * new * heads * d * (size + 1) + 8 * touched * heads + 4 * touched + 2 * rows * d * size + (4 * new if c["moved"] else 0)
        return {"bytes": float(moved), "flops": float(3 * new * heads * (group + 1) * c["rotary"] + 2 * new * heads * d)}
    if c["kind"] == "bound":
        reach = sum(t - (t - m) // bs * bs for m, t in n)
        return {"bytes": float(heads * d * (reach + 2 * touched) + 4 * touched), "flops": float(2 * heads * d * reach)}
    if c["kind"] == "select":
        # blocks that are neither taken nor left out unseen
        scored = [[max(0, b - c["first"] - c["recent"]) if b > c["select"] else 0 for b in ((t - m + i) // bs + 1 for i in range(m))] for m, t in n]
        reads = sum(max(x) for x in scored)
        return {"bytes": float(heads * reads * (2 * d + 4) + 4 * reads + (rows * d * size if reads else 0) + 4 * new * heads * c["select"]),
                "flops": float(4 * d * heads * group * sum(map(sum, scored)))}
    if c["kind"] == "blocks":
        reads = pairs = 0
        for m, t in n:
            each = [min((t - m + i) // bs + 1, c["select"]) for i in range(m)]
            reads += min(-(-t // bs), max(each))
            pairs += sum(min(x * bs, t - m + i + 1) for i, x in enumerate(each))
        return {"bytes": float(heads * reads * (2 * bs * d + 8) + 4 * reads + 4 * new * heads * c["select"] + rows * (2 * d * size + 4)),
                "flops": float(4 * d * heads * group * pairs)}
    once = tokens
    first = 0
    for end, p in _prefixes(c):
        once -= p // bs * bs * (end - first - 1)
        first = end
    pairs = sum(m * t - m * (m - 1) // 2 for m, t in n)
    return {"bytes": float(2 * once * heads * d + 8 * (once // bs) * heads + 4 * once // bs + rows * (2 * d * size + 4)), "flops": float(4 * d * heads * group * pairs)}


# ------------------------------------------------------------------ inputs
def _codes(gen, c, blocks):
    """e4m3 numbers of normal values, some channels larger than the rest, [blocks, slots, heads, dim]."""
    shape = (blocks, c["block"], c["heads"], c["dim"]) if c["order"] == "slots" else (blocks, c["heads"], c["block"], c["dim"])
    x = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16) * 64
    x[..., ::37] *= 1.6
    x = x.clamp_(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
    return x if c["order"] == "slots" else x.transpose(1, 2)


def _scales(gen, c, blocks):
    return torch.randint(-7, -4, (blocks, c["heads"]), generator=gen, device=DEV).float().exp2()


def _rows_of(gen, c, total, count, dtype, spread=1.0):
    """[total, count, dim] values, the first of `count` groups of heads in a wider row where a fused projection made them."""
    wide = count + (2 if c["fused"] else 0) * c["heads"]
    x = torch.randn((total, wide, c["dim"]), generator=gen, device=DEV, dtype=torch.float32 if dtype == "fp32" else torch.bfloat16)
    x = (x * spread).to(TORCH[dtype])
    x[..., ::37] *= 3
    return x


def prepare(case, seed):
    c, gen, r = case, torch.Generator(device=DEV).manual_seed(seed), random.Random(seed)
    n = _lengths(c)
    if c["kind"] != "shared":
        r.shuffle(n)
    total, per = sum(m for m, _ in n), -(-_most(c) // c["block"])
    bs, heads, dim, dtype = c["block"], c["heads"], c["dim"], TORCH[c["dtype"]]
    s = {"case": c, "total": total, "most_new": max(m for m, _ in n), "most": max(t for _, t in n), "rows": None, "starts": None,
         "k": _codes(gen, c, c["seqs"] * per), "k_scale": _scales(gen, c, c["seqs"] * per),
         "table": torch.randperm(c["seqs"] * per, generator=gen, device=DEV).to(torch.int32).view(c["seqs"], per),
         "lens": torch.tensor([t for _, t in n], dtype=torch.int32, device=DEV)}
    s["v"], s["v_scale"] = _codes(gen, c, c["seqs"] * per), _scales(gen, c, c["seqs"] * per)
    rows = sorted(r.sample(range(c["seqs"]), c["reqs"]))
    if c["seqs"] != c["reqs"]:
        s["rows"] = torch.tensor(rows, dtype=torch.int32, device=DEV)
    starts = [0]
    for m, _ in n:
        starts.append(starts[-1] + m)
    if any(m != 1 for m, _ in n):
        s["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    if c["kind"] == "rotate":
        if c["fused"]:
            x = _rows_of(gen, c, total, heads * c["group"], c["dtype"])
            s["q"], s["key"], s["value"] = x[:, :-2 * heads], x[:, -2 * heads:-heads], x[:, -heads:]
        else:
            s["q"] = _rows_of(gen, c, total, heads * c["group"], c["dtype"])
            s["key"], s["value"] = (_rows_of(gen, c, total, heads, c["dtype"]) for _ in range(2))
        s["rotated"] = torch.empty((total, heads * c["group"], dim), dtype=dtype, device=DEV)
        pairs = torch.arange(c["rotary"] // 2, device=DEV, dtype=torch.float64)
        s["freq"] = (500000.0 ** (-2 * pairs / c["rotary"])).float()
        s["positions"] = None
        if c["moved"]:                          # what each request has lost of its context
            at = torch.cat([torch.arange(t - m, t) + r.randint(0, c["moved"]) for m, t in n])
            s["positions"] = at.to(torch.int32).to(DEV)
    elif c["kind"] in ("bound", "select"):
        s["bounds"] = torch.zeros((c["seqs"] * per, heads, 2, dim), dtype=torch.float8_e4m3fn, device=DEV)
        if c["kind"] == "select":
            # the least and the largest of a block, as bound() leaves them: normal values' largest of so many lie about there
            top = math.sqrt(2 * math.log(bs)) * 64
            x = top + 16 * torch.randn((c["seqs"] * per, heads, 2, dim), generator=gen, device=DEV, dtype=torch.bfloat16)
            x += 24 * torch.randn((c["seqs"] * per, heads, 1, dim), generator=gen, device=DEV, dtype=torch.bfloat16)
            x[:, :, 0] *= -1
            s["bounds"] = torch.sort(x, dim=2).values.clamp_(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
            s["blocks"] = torch.empty((total, heads, c["select"]), dtype=torch.int32, device=DEV)
    elif c["kind"] == "blocks":
        # for each token and head: the first and the newest blocks, and others, in order
        last = torch.cat([torch.arange(t - m, t) for m, t in n]).to(DEV) // bs
        width = max(-(-s["most"] // bs), c["select"])
        at = torch.arange(width, device=DEV)
        s["blocks"] = torch.empty((total, heads, c["select"]), dtype=torch.int32, device=DEV)
        step = max(1, (1 << 26) // (heads * width))
        for i in range(0, total, step):
            end = last[i:i + step, None, None]
            key = torch.rand((len(end), heads, width), generator=gen, device=DEV)
            key = torch.where((at < c["first"]) | (at > end - c["recent"]), 2.0, key)
            key = torch.where(at > end, -1.0, key)
            taken = torch.topk(key, c["select"], dim=-1)
            taken = torch.where(taken.values < 0, width, taken.indices).sort(-1).values
            s["blocks"][i:i + step] = torch.where(taken == width, -1, taken)
    else:
        first, firsts = 0, [0]
        for end, p in _prefixes(c):             # the members' rows begin with the same blocks
            s["table"][rows[first:end], :p // bs] = s["table"][rows[first], :p // bs].clone()
            firsts.append(end)
            first = end
        s["group_starts"] = torch.tensor(firsts, dtype=torch.int32, device=DEV)
        s["prefix"] = torch.tensor([p for _, p in _prefixes(c)], dtype=torch.int32, device=DEV)
    if c["kind"] in ("select", "blocks", "shared"):
        s["q"] = _rows_of(gen, c, total, heads * c["group"], c["dtype"], 1.2)[:, :heads * c["group"]]
    if c["kind"] in ("blocks", "shared"):
        s["out"] = torch.empty((total, heads * c["group"], dim), dtype=dtype, device=DEV)
        s["lse"] = torch.empty((total, heads * c["group"]), dtype=torch.float32, device=DEV)
    return s


# ------------------------------------------------------------------ one pass: the framework's operators
def _handle(s):
    """The cache's and the batch's descriptions, which a serving loop makes once."""
    if "cache" not in s:
        from paper_2605_11093_amd import binding as B
        c = s["case"]
        s["cache"] = B.KV8(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"])
        s["batch"] = B.KV8Batch(s["lens"], starts=s["starts"], rows=s["rows"], total_new=s["total"], max_new=s["most_new"],
                                max_len=s["most"])
        if c["kind"] == "rotate":
            s["rotary"] = B.KV8Rotary(s["freq"], positions=s["positions"], pairs=c["pairs"])
        if c["kind"] == "shared":
            s["shares"] = B.KV8Prefix(s["group_starts"], s["prefix"], max_prefix=c["prefix_hi"])
        s["B"] = B
    return s["B"], torch.cuda.current_stream().cuda_stream


def _run_own(s):
    c = s["case"]
    B, stream = _handle(s)
    if c["kind"] == "rotate":
        B.kv8_append_rotated(s["cache"], s["batch"], s["key"], s["value"], s["rotary"], q=s["q"], q_out=s["rotated"], stream=stream)
        return {k: s[k] for k in ("k", "v", "k_scale", "v_scale", "rotated")}
    if c["kind"] == "bound":
        B.kv8_bound(s["cache"], s["batch"], s["bounds"], stream=stream)
        return {"bounds": s["bounds"]}
    if c["kind"] == "select":
        B.kv8_select(s["cache"], s["batch"], s["bounds"], s["q"], s["blocks"], first=c["first"], recent=c["recent"], stream=stream)
        return {"blocks": s["blocks"]}
    if c["kind"] == "blocks":
        B.kv8_attend_blocks(s["cache"], s["batch"], s["blocks"], s["q"], s["out"], lse=s["lse"], stream=stream)
    else:
        B.kv8_attend_shared(s["cache"], s["batch"], s["shares"], s["q"], s["out"], lse=s["lse"], stream=stream)
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------ the same, plainly
def _e4m3(x):
    return torch.where(x.isnan(), x, x.clamp(-LARGEST, LARGEST)).to(torch.float8_e4m3fn)


def _bytes(x):
    return x.view(torch.uint8)


def _who(s):
    """(request, position) of every new token, the table's rows in the requests' order, where new rows start, the lengths."""
    table = s["table"] if s["rows"] is None else s["table"][s["rows"].long()]
    lens = s["lens"].long()
    starts = torch.arange(len(lens) + 1, device=DEV) if s["starts"] is None else s["starts"].long()
    at = torch.arange(s["total"], device=DEV)
    req = torch.searchsorted(starts, at, right=True) - 1
    return req, lens[req] - starts[req + 1] + at, table, starts, lens


def _turned(x, cos, sin, pairs):
    """x [rows, heads, dim] in 64 bits, its first elements rotated, rounded to single precision."""
    half = cos.shape[-1]
    x, cos, sin = x.double(), cos[:, None], sin[:, None]
    a, b = (x[..., :2 * half:2], x[..., 1:2 * half:2]) if pairs else (x[..., :half], x[..., half:2 * half])
    a, b = a * cos - b * sin, a * sin + b * cos
    front = torch.stack((a, b), -1).flatten(-2) if pairs else torch.cat((a, b), -1)
    return torch.cat((front, x[..., 2 * half:]), -1).float()


def _rotate(s):
    c = s["case"]
    bs = c["block"]
    req, pos, table, starts, lens = _who(s)
    angle = (pos if s["positions"] is None else s["positions"].long()).double()[:, None] * s["freq"].double()
    cos, sin = angle.cos().float().double(), angle.sin().float().double()
    s["rotated"].copy_(_turned(s["q"], cos, sin, c["pairs"]))
    new = starts[1:] - starts[:-1]
    first = lens - new                                              # the first new token's position
    # the blocks a request touches lie in a row of a grid
    wide = (s["most_new"] + bs - 2) // bs + 2
    cell = req * wide + pos // bs - first[req] // bs
    block = table[req, pos // bs].long()
    inside = first % bs                                             # older tokens in its first block
    older = (torch.arange(bs, device=DEV) < inside[:, None]) & (new > 0)[:, None]
    firsts = table[torch.arange(len(lens), device=DEV), (first // bs).clamp(max=table.shape[1] - 1)].long()
    for name, x in (("k", _turned(s["key"], cos, sin, c["pairs"])), ("v", s["value"].float())):
        codes, scale = s[name], s[name + "_scale"]
        grid = torch.zeros((len(lens) * wide, c["heads"]), device=DEV)
        largest = x.abs().amax(-1)                                                          # [total, heads]
        grid.scatter_reduce_(0, cell[:, None].expand_as(largest), largest, "amax")
        mantissa, exponent = torch.frexp(grid / LARGEST)
        exponent = torch.where(mantissa == 0.5, exponent - 1, exponent)
        exponent = torch.where(grid > 0, exponent, -100).clamp(min=-100)
        need = ((exponent + 127) << 23).to(torch.int32).view(torch.float32).view(len(lens), wide, -1)     # 2 ** exponent
        had = scale[firsts]
        begun = (inside > 0) & (new > 0)
        need[:, 0] = torch.where(begun[:, None], torch.maximum(need[:, 0], had), need[:, 0])
        # what the first block holds already
        old = codes[firsts].float() * (had / need[:, 0])[:, None, :, None]
        request, slot = older.nonzero(as_tuple=True)
        _bytes(codes)[firsts[request], slot] = _bytes(_e4m3(old[request, slot]))
        need = need.view(-1, c["heads"])[cell]
        scale[block] = need
        _bytes(codes)[block, pos % bs] = _bytes(_e4m3(x / need[:, :, None]))
    return {k: s[k] for k in ("k", "v", "k_scale", "v_scale", "rotated")}


def _bound(s):
    c = s["case"]
    bs, blocks = c["block"], -(-s["most"] // c["block"])
    _, _, table, starts, lens = _who(s)
    begin = lens - (starts[1:] - starts[:-1])
    j = torch.arange(blocks, device=DEV)
    request, j = ((j >= (begin // bs)[:, None]) & (j * bs < lens[:, None])).nonzero(as_tuple=True)     # the touched blocks
    at = table[request, j].long()
    x = _bytes(s["k"])[at].view(torch.float8_e4m3fn).float()                                # [touched, slots, heads, dim]
    there = (torch.arange(bs, device=DEV) < (lens[request] - j * bs)[:, None])[:, :, None, None]
    low, high = torch.where(there, x, math.inf).amin(1), torch.where(there, x, -math.inf).amax(1)
    _bytes(s["bounds"])[at] = _bytes(torch.stack((low, high), 2).to(torch.float8_e4m3fn))
    return {"bounds": s["bounds"]}


def _select(s):
    c = s["case"]
    bs, heads, group, dim = c["block"], c["heads"], c["group"], c["dim"]
    req, pos, table, starts, _ = _who(s)
    last, blocks, n = pos // bs, -(-s["most"] // bs), c["reqs"]
    # scores in 64 bits: which of two blocks has the larger one may hang on the last bit
    entry = table[:, :blocks].long()
    b = _bytes(s["bounds"])[entry].view(torch.float8_e4m3fn).permute(0, 2, 3, 4, 1).double()   # [requests, heads, 2, dim, blocks]
    at = (starts[:-1, None] + torch.arange(s["most_new"], device=DEV)).clamp(max=s["total"] - 1)
    q = s["q"][at].double().view(n, -1, heads, group, dim).transpose(1, 2).reshape(n, heads, -1, dim)
    z = torch.matmul(q.clamp(max=0), b[:, :, 0].contiguous())
    z += torch.matmul(q.clamp(min=0), b[:, :, 1].contiguous())
    z = z.view(n, heads, -1, group, blocks).amax(3) * s["k_scale"][entry].double().transpose(1, 2)[:, :, None]
    j = torch.arange(max(blocks, c["select"]), device=DEV)
    score = torch.full((s["total"], heads, len(j)), -math.inf, dtype=torch.float64, device=DEV)
    score[:, :, :blocks] = z[req, :, torch.arange(s["total"], device=DEV) - starts[req]]
    end = last[:, None, None]
    score = torch.where((j < c["first"]) | (j > end - c["recent"]), math.inf, score)
    score = torch.where(j > end, -math.inf, score)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :c["select"]]
    order = torch.where(order > end, len(j), order).sort(-1).values
    s["blocks"].copy_(torch.where(order == len(j), -1, order))
    return {"blocks": s["blocks"]}


def _softmax_out(s, p, v, shape):
    """p: scores, -inf where hidden, [..., rows, tokens]; v [..., tokens, dim].  Outputs and log-sum-exp, of `shape` rows."""
    p *= 1.0 / math.sqrt(s["case"]["dim"])
    top = p.amax(-1, keepdim=True)
    top = torch.where(top.isfinite(), top, 0.0)
    p -= top
    p.exp_()
    total = p.sum(-1, keepdim=True)
    p /= torch.where(total > 0, total, 1.0)
    return torch.matmul(p, v).view(*shape, -1), (top + total.log()).view(shape)


def _attend_blocks(s):
    c = s["case"]
    bs, heads, group, dim, total = c["block"], c["heads"], c["group"], c["dim"], s["total"]
    req, pos, table, _, _ = _who(s)
    listed_blocks = s["blocks"].long()                                                      # [total, heads, select]
    entry = table[req[:, None, None], listed_blocks.clamp(min=0)].long()
    head = torch.arange(heads, device=DEV)[:, None]
    at = listed_blocks[..., None] * bs + torch.arange(bs, device=DEV)
    hidden = ((listed_blocks < 0)[..., None] | (at > pos[:, None, None, None])).flatten(2)[:, :, None]
    k, v = (_bytes(s[x]).permute(0, 2, 1, 3)[entry, head].view(torch.float8_e4m3fn).float().mul_(s[x + "_scale"][entry, head][..., None, None]).flatten(2, 3)
            for x in ("k", "v"))                                                            # [total, heads, tokens, dim]
    p = torch.matmul(s["q"].float().reshape(total, heads, group, dim), k.transpose(2, 3).contiguous())
    p.masked_fill_(hidden, -math.inf)
    out, lse = _softmax_out(s, p, v, (total, heads, group))
    s["out"].copy_(out.view(s["out"].shape))
    s["lse"].copy_(lse.view(s["lse"].shape))
    return {"out": s["out"], "lse": s["lse"]}


def _gathered(codes, scale, table):
    """[requests, heads, tokens, dim] in single precision."""
    x = _bytes(codes)[table.long()].view(torch.float8_e4m3fn).float()                       # [n, blocks, slots, heads, dim]
    x *= scale[table.long()][:, :, None, :, None]
    return x.flatten(1, 2).transpose(1, 2)


def _attend_shared(s):
    c = s["case"]
    heads, group, most_new, n = c["heads"], c["group"], s["most_new"], c["reqs"]
    _, _, table, starts, lens = _who(s)
    table = table[:, :-(-s["most"] // c["block"])]
    new = starts[1:] - starts[:-1]
    i = torch.arange(most_new, device=DEV)
    at = (starts[:-1, None] + i).clamp(max=s["total"] - 1)
    q = s["q"][at].float().view(n, most_new, heads, group, c["dim"]).transpose(1, 2).reshape(n, heads, most_new * group, c["dim"])
    k = _gathered(s["k"], s["k_scale"], table).transpose(2, 3).contiguous()
    p = torch.matmul(q, k).view(n, heads, most_new, group, -1)
    del k
    seen = torch.arange(p.shape[-1], device=DEV) <= (lens - new)[:, None, None] + i[:, None]
    seen &= (i < new[:, None])[:, :, None]
    p.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    v = _gathered(s["v"], s["v_scale"], table).contiguous()
    out, lse = _softmax_out(s, p.flatten(2, 3), v, (n, heads, most_new, group))
    valid = i < new[:, None]
    s["out"].copy_(out.permute(0, 2, 1, 3, 4)[valid].reshape(s["out"].shape))
    s["lse"].copy_(lse.permute(0, 2, 1, 3)[valid].reshape(s["lse"].shape))
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    if own:
        return _run_own(state)
    return {"rotate": _rotate, "bound": _bound, "select": _select, "blocks": _attend_blocks, "shared": _attend_shared}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ the same in 64 bits
def _numbers():
    """What the 256 codes stand for."""
    out = []
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        x = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        out.append(math.nan if code & 127 == 127 else -x if code & 128 else x)
    return torch.tensor(out, dtype=torch.float64, device=DEV)


def _nearest(x):
    """The nearest e4m3 number to each of x, ties to even, in 64 bits."""
    size = x.abs().clamp(max=448.0)
    steps = torch.tensor([2.0 ** (e - 3) for e in range(-6, 9)], dtype=torch.float64, device=DEV)
    step = steps[((torch.frexp(size).exponent - 1).clamp(min=-6) + 6).long()]
    return torch.copysign(torch.round(size / step) * step, x)


def _spans(s):
    """(request, its row of the table, where its new rows start, how many, its length), on the host."""
    lens = s["lens"].tolist()
    rows = list(range(len(lens))) if s["rows"] is None else s["rows"].tolist()
    starts = list(range(len(lens) + 1)) if s["starts"] is None else s["starts"].tolist()
    return [(r, rows[r], starts[r], starts[r + 1] - starts[r], lens[r]) for r in range(len(lens))]


def _exact_turn(x, position, freq, pairs):
    """A complex product for every pair of elements, by factors whose parts have been rounded to single precision."""
    angle = position.double()[:, None] * freq.double()
    factor = torch.complex(torch.cos(angle).float().double(), torch.sin(angle).float().double())[:, None]
    x, m = x.double(), freq.shape[0]
    first, second = (torch.arange(m, device=DEV) * 2, torch.arange(m, device=DEV) * 2 + 1) if pairs else (torch.arange(m, device=DEV), torch.arange(m, device=DEV) + m)
    z = torch.complex(x[..., first], x[..., second]) * factor
    x = x.clone()
    x[..., first], x[..., second] = z.real.clone(), z.imag.clone()
    return x


def _exact_rotate(s):
    c, number = s["case"], _numbers()
    bs, out = c["block"], {}
    table = s["table"].tolist()
    where, position = [], []                                        # (block, first slot, slots, first row) of every touched block
    for _, row, start, new, length in _spans(s):
        p = length - new
        position += range(p, length)
        while p < length:
            m = min(bs - p % bs, length - p)
            where.append((table[row][p // bs], p % bs, m, start + p - (length - new)))
            p += m
    position = torch.tensor(position, device=DEV) if s["positions"] is None else s["positions"]
    t = torch.tensor(where, device=DEV)
    slot = torch.arange(bs, device=DEV)
    key = _exact_turn(s["key"], position, s["freq"], c["pairs"]).float()                    # (the definition rounds it)
    for name, x in (("k", key), ("v", s["value"])):
        all_codes = number[s[name].view(torch.uint8).int()]
        scales = s[name + "_scale"].double()
        fresh = (slot >= t[:, 1:2]) & (slot < t[:, 1:2] + t[:, 2:3])
        source = (t[:, 3:4] + slot - t[:, 1:2]).clamp(0, s["total"] - 1)
        rows = torch.where(fresh[..., None, None], x[source].double(), 0.0)
        most = rows.abs().amax((1, 3))
        power = torch.ceil(torch.log2(most.clamp(min=1e-300) / 448.0))
        for wrong in (-1, 1):                                       # the logarithm is rounded: its neighbours decide
            power = torch.where((most <= 448.0 * torch.exp2(power - 1)) if wrong < 0 else (most > 448.0 * torch.exp2(power)), power + wrong, power)
        scale = torch.exp2(power.clamp(min=-100.0))
        had = scales[t[:, 0]]
        scale = torch.where(t[:, 1:2] > 0, torch.maximum(scale, had), scale)
        block = all_codes[t[:, 0]]
        older = _nearest(block * (had / scale)[:, None, :, None])
        block = torch.where((slot < t[:, 1:2])[..., None, None], older, block)
        block = torch.where(fresh[..., None, None], _nearest(rows / scale[:, None, :, None]), block)
        all_codes[t[:, 0]] = block
        scales[t[:, 0]] = scale
        out[name], out[name + "_scale"] = all_codes, scales
    return {**{k: out[k] for k in ("k", "v", "k_scale", "v_scale")}, "rotated": _exact_turn(s["q"], position, s["freq"], c["pairs"])}


def _exact_bound(s):
    c, number = s["case"], _numbers()
    got = number[s["bounds"].view(torch.uint8).int()]
    for _, row, _, new, length in _spans(s):
        first = (length - new) // c["block"]
        at = s["table"][row, first:-(-length // c["block"])].long()
        x = number[s["k"].view(torch.uint8)[at].int()]
        for low, fill in ((0, math.inf), (1, -math.inf)):
            y = x.clone()
            rest = length - first * c["block"]
            y.view(-1, c["heads"], c["dim"])[rest:] = fill
            got[at, :, low] = y.max(1).values if low else y.min(1).values
    return {"bounds": got}


def _exact_select(s):
    c, number = s["case"], _numbers()
    heads, group, bs = c["heads"], c["group"], c["block"]
    out = torch.full(s["blocks"].shape, -1, dtype=torch.int32, device=DEV)
    for _, row, start, new, length in _spans(s):
        entry = s["table"][row, :-(-length // bs)].long()
        b = number[s["bounds"].view(torch.uint8)[entry].int()]                              # [blocks, heads, 2, dim]
        for i in range(new):
            end = (length - new + i) // bs + 1
            if end <= c["select"]:
                out[start + i, :, :end] = torch.arange(end, dtype=torch.int32, device=DEV)
                continue
            score = torch.full((heads, end), -math.inf, dtype=torch.float64, device=DEV)
            for g in range(group):
                q = s["q"][start + i, g::group].double()[None, :, None]                     # heads that share one are neighbours
                score = torch.maximum(score, torch.maximum(q * b[:end, :, :1], q * b[:end, :, 1:]).sum((2, 3)).t())
            score *= s["k_scale"][entry[:end]].double().t()
            middle = score[:, c["first"]:end - c["recent"]]
            wanted = c["select"] - c["first"] - c["recent"]
            taken = torch.argsort(middle, dim=-1, descending=True, stable=True)[:, :wanted].sort(-1).values + c["first"]
            edge = torch.arange(end, device=DEV).expand(heads, -1)
            out[start + i] = torch.cat((edge[:, :c["first"]], taken, edge[:, end - c["recent"]:]), -1)
    return {"blocks": out}


def _exact_rows(q, k, v, hidden, dim):
    z = torch.matmul(q, k.t().contiguous()) / math.sqrt(dim)
    z.masked_fill_(hidden, -math.inf)
    total = torch.logsumexp(z, -1)
    return torch.matmul(torch.exp(z - total[..., None]), v), total


def _exact_blocks(s):
    c, number = s["case"], _numbers()
    heads, group, d, bs = c["heads"], c["group"], c["dim"], c["block"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    listed_blocks = s["blocks"].tolist()
    if s["total"] * heads > 4000:
        return None
    for _, row, start, new, length in _spans(s):
        for i in range(start, start + new):
            seen = length - new + i - start + 1
            for h in range(heads):
                own_list = torch.tensor([b for b in listed_blocks[i][h] if b >= 0], device=DEV)
                at = s["table"][row].long()[own_list]
                k, v = ((number[s[x].view(torch.uint8)[at, :, h].int()] * s[x + "_scale"][at, h].double()[:, None, None]).flatten(0, 1) for x in ("k", "v"))
                hidden = (own_list[:, None] * bs + torch.arange(bs, device=DEV)).flatten() >= seen
                rows = slice(h * group, (h + 1) * group)
                out[i, rows], lse[i, rows] = _exact_rows(s["q"][i, rows].double(), k, v, hidden, d)
    return {"out": out, "lse": lse}


def _exact_shared(s):
    c, number = s["case"], _numbers()
    heads, group, d, bs = c["heads"], c["group"], c["dim"], c["block"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    for _, row, start, new, length in _spans(s):
        blocks = s["table"][row, :-(-length // bs)].long()
        k, v = (number[s[x].view(torch.uint8)[blocks].int()] * s[x + "_scale"][blocks].double()[:, None, :, None] for x in ("k", "v"))
        k, v = (x.flatten(0, 1)[:length].transpose(0, 1).contiguous() for x in (k, v))                # [heads, length, d]
        hidden = torch.arange(length, device=DEV) > length - new + torch.arange(new, device=DEV)[:, None]
        for h in range(heads):
            rows = slice(h * group, (h + 1) * group)
            q = s["q"][start:start + new, rows].double().transpose(0, 1).reshape(-1, d)                # [group * new, d]
            o, total = _exact_rows(q, k[h], v[h], hidden.repeat(group, 1), d)
            out[start:start + new, rows] = o.view(group, new, d).transpose(0, 1)
            lse[start:start + new, rows] = total.view(group, new).t()
    return {"out": out, "lse": lse}


def exact(case, seed):
    kinds = {"rotate": _exact_rotate, "bound": _exact_bound, "select": _exact_select, "blocks": _exact_blocks, "shared": _exact_shared}
    return kinds[case["kind"]](prepare(case, seed))
