"""The operators between the linear layers of a block, as cases that can be timed.

Four operators of `paper_2501_07139_b200`, in the order in which a serving step uses them:

  blocks     `fq_cache_step`: every sequence's cache is cut back to `keep` tokens and grows by `new` ones; blocks go back to and come from a
             free list; where each new token is stored, its position, and for a drafted tree which of the new tokens it sees
  rotary     `fq_rotary`, `fq_rotary_cache`: queries and keys are turned by angles that grow with the token's position; the second stores
             keys and values in the cache as well
  attention  `fq_tree_attention`: a sequence's new tokens see what is cached and, of the new tokens, those of a tree's branch (mask "tree") or
             those before them ("chain")
  move       `fq_cache_move`: the accepted branch of a tree is moved to the end of what is kept, in the caches of all layers

Where the module's `own` is false the same results come from elementary torch operations.  Heads of 128 are those of this repository's
7B and 13B stacks (32 and 40 of them); shared key heads, other head sizes, blocks and lengths are generic.
"""
import math

import torch

own = False

FQ = None                                # the library context that a serving program keeps


def context():
    global FQ
    if FQ is None:
        import paper_2501_07139_b200 as P
        FQ = P.FlexQ(1)
    return FQ


TABLES = {}                              # the tables of angles that it keeps, one for each way of turning


def turns(case):
    kind = case["rot"], case["scaled"]
    if kind not in TABLES:
        import paper_2501_07139_b200 as P
        TABLES[kind] = P.fq_rotary_table(case["rot"], 10000.0, **(SCALING if case["scaled"] else {}), device="cuda")
    return TABLES[kind]


DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # a step's bookkeeping for a batch whose sequences each have a drafted tree; the last step accepted some of the tree before it
        {"name": "blocks-64-trees", "op": "blocks", "seqs": 64, "new": 24, "context": 4096, "block": 16, "tree": True},
        # prompts take the place of finished requests, among some hundred that go on
        {"name": "blocks-300-prompts", "op": "blocks", "seqs": 300, "new": 3000, "context": 8000, "block": 32, "tree": False},
        # one token of the 7B stack: its latency in a decode step
        {"name": "rotary-1x32-cache", "op": "rotary", "tokens": 1, "heads": 32, "kv": 32, "dim": 128, "rot": 128, "type": "fp16", "pairs": "half",
         "far": 4096, "scaled": False, "pass": "cache"},
        # a ragged prompt far into a long context, shared key heads, half of the head turned, frequencies scaled by parts
        {"name": "rotary-777x48-cache", "op": "rotary", "tokens": 777, "heads": 48, "kv": 8, "dim": 128, "rot": 64, "type": "bf16", "pairs": "interleaved",
         "far": 1000000, "scaled": True, "pass": "cache"},
        # the gradient of four calibration sequences through the 13B stack's queries and keys
        {"name": "rotary-8192x40-gradient", "op": "rotary", "tokens": 8192, "heads": 40, "kv": 40, "dim": 128, "rot": 128, "type": "fp32", "pairs": "half",
         "far": 2048, "scaled": False, "pass": "gradient"},
        # one sequence, one token: the latency of a decode step of the 7B stack
        {"name": "attention-1x1x4000", "op": "attention", "seqs": 1, "new": 1, "context": 4000, "heads": 32, "kv": 32, "dim": 128, "block": 16,
         "type": "fp16", "mask": "chain"},
        # a batch of the 13B stack decoded together, ragged
        {"name": "attention-48x1x4096", "op": "attention", "seqs": 48, "new": 1, "context": 4096, "heads": 40, "kv": 40, "dim": 128, "block": 32,
         "type": "bf16", "mask": "chain"},
        # drafted trees of eight tokens (what a batched decode call takes), shared key heads, ragged
        {"name": "attention-16x8x16000", "op": "attention", "seqs": 16, "new": 8, "context": 16000, "heads": 32, "kv": 8, "dim": 128, "block": 16,
         "type": "bf16", "mask": "tree"},
        # trees of sixty tokens over long contexts: many rows share a key head
        {"name": "attention-5x60x40000", "op": "attention", "seqs": 5, "new": 60, "context": 40000, "heads": 64, "kv": 8, "dim": 128, "block": 64,
         "type": "bf16", "mask": "tree"},
        # calibration sequences through a block of the 7B stack, nothing cached before
        {"name": "attention-4x2048x0", "op": "attention", "seqs": 4, "new": 2048, "context": 0, "heads": 32, "kv": 32, "dim": 128, "block": 128,
         "type": "bf16", "mask": "chain"},
        # the accepted branch of one tree of eight, all layers of the 7B stack
        {"name": "move-1x8x32", "op": "move", "seqs": 1, "new": 8, "layers": 32, "kv": 32, "dim": 128, "context": 2000, "block": 16, "type": "fp16"},
        # a batch of larger trees, shared key heads
        {"name": "move-90x40x32", "op": "move", "seqs": 90, "new": 40, "layers": 32, "kv": 8, "dim": 128, "context": 200, "block": 16, "type": "bf16"},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], evenly spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("blocks", "rotary", "attention", "attention", "move"))
    block = rng.choice((8, 16, 16, 32, 64, 100, 128))
    if op == "blocks":
        tree = rng.random() < 0.5
        new, seqs = (_spread(rng, 1, 64), _spread(rng, 1, 1000)) if tree else (_spread(rng, 1, 4096), _spread(rng, 1, 1000))
        return {"op": op, "seqs": min(seqs, max(1, 900000 // new)), "new": new, "context": _spread(rng, 1, 16384), "block": block, "tree": tree}
    kv, dim = rng.choice((1, 2, 4, 8, 8, 32, 40)), rng.choice((64, 80, 96, 128, 128, 128, 256))
    heads = kv * rng.choice((1, 1, 4, 7, 8) if kv <= 8 else (1,))
    if op == "rotary":
        kind = rng.choice(("bf16", "fp16", "fp32"))
        return {"op": op, "tokens": min(_spread(rng, 1, 16384), 320_000_000 // ((heads + kv) * dim * SIZE[kind])), "heads": heads, "kv": kv, "dim": dim,
                "rot": rng.choice((dim, dim, dim // 2)), "type": kind, "pairs": rng.choice(("half", "interleaved")), "far": _spread(rng, 1, 1000000),
                "scaled": rng.random() < 0.5, "pass": rng.choice(("cache", "apart", "gradient"))}
    kind = rng.choice(("bf16", "bf16", "fp16"))
    if op == "move":
        new, context = _spread(rng, 2, 64), _spread(rng, 1, 2000)
        most = 1_000_000_000 // (2 * (context + new + block) * kv * dim)         # layers times sequences
        layers = min(_spread(rng, 1, 40), most)
        seqs = min(_spread(rng, 1, 90), most // layers)
        return {"op": op, "seqs": seqs, "new": new, "layers": layers, "kv": kv, "dim": dim, "context": context, "block": block, "type": kind}
    mask = rng.choice(("tree", "chain"))
    new = rng.choice((1, 1, _spread(rng, 1, 64), _spread(rng, 1, 64), _spread(rng, 1, 2048)))
    new = min(new, 64) if mask == "tree" else min(new, math.isqrt(36_000_000_000 // (heads * dim)))
    context = min(_spread(rng, 1, 40000), 500_000_000 // (kv * dim), 40_000_000_000 // (new * heads * dim) - new)
    seqs = min(_spread(rng, 1, 64), max(1, 500_000_000 // ((context + new) * kv * dim)), max(1, 40_000_000_000 // ((context + new) * new * heads * dim)))
    return {"op": op, "seqs": seqs, "new": new, "context": context, "heads": heads, "kv": kv, "dim": dim, "block": block, "type": kind, "mask": mask}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _ragged(case):
    """Every sequence's cached and new tokens: the first has all of `context` and `new`, others between nothing and that."""
    cached = [int(case["context"] * (1.0 - b * 0.6180339887 % 1.0)) for b in range(case["seqs"])]
    new = [max(1, round(case["new"] * (1.0 - b * 0.7548776662 % 1.0))) for b in range(case["seqs"])]
    if case["new"] > 1:
        new[7::9] = [0] * len(new[7::9])                # a sequence that waits
    return cached, new


def _table(seqs, lens, block, width, blocks, g):
    """Block tables [seqs][width] of sequences of `lens` tokens, and the blocks that are left, in an order as a running server has it."""
    order = torch.randperm(blocks, device="cuda", generator=g, dtype=torch.int32)
    have = (lens + block - 1) // block
    first = torch.cumsum(have, 0) - have
    col = torch.arange(width, device="cuda")
    held = col[None] < have[:, None]
    table = torch.where(held, order[(first[:, None] + col[None]).clamp(max=blocks - 1)], -1).to(torch.int32)
    return table, order.flip(0), int(have.sum())


def _parents(new, g):
    """A drafted tree for every sequence: the parent of token i is one before it, often the one right before; the first has none."""
    total = int(new.sum())
    i = torch.arange(total, device="cuda") - torch.repeat_interleave(torch.cumsum(new, 0) - new, new)
    before = torch.minimum((torch.rand(total, device="cuda", generator=g) * i).long(), i - 1)
    return torch.where(torch.rand(total, device="cuda", generator=g) < 0.5, i - 1, before).to(torch.int32)


def _closure(parents, starts, words):
    """For every new token: which new tokens of its sequence are itself or above it, as bits, and how many are above it."""
    total = parents.shape[0]
    row = torch.arange(total, device=parents.device)
    seq = torch.searchsorted(starts[1:].contiguous(), row, right=True)
    first = starts[seq].long()
    up = torch.where(parents >= 0, first + parents, total)              # the token above; `total`: none
    up = torch.cat((up, up.new_tensor([total])))
    seen = torch.zeros((total + 1, words * 64), dtype=torch.bool, device=parents.device)
    seen[row, row - first] = True
    depth = torch.cat((torch.ones_like(row), row.new_zeros(1)))         # tokens on the way up so far, this one among them
    for _ in range(max(1, (words * 64 - 1).bit_length())):              # ways twice as long each time
        seen, depth, up = seen | seen[up], depth + depth[up], up[up]
    bits = (seen[:total].view(total, words, 64).long() << torch.arange(64, device=parents.device)).sum(2)
    return bits, depth[:total] - 1


def _frequencies(case, device):
    """Radians a position, in 64 bits; scaled by parts: what turns less than `low` times in the original context is slowed by `factor`."""
    f = 10000.0 ** (-2.0 * torch.arange(case["rot"] // 2, dtype=torch.float64, device=device) / case["rot"])
    if not case["scaled"]:
        return f
    turns = SCALING["context"] * f / (2 * math.pi)
    keep = ((turns - SCALING["low"]) / (SCALING["high"] - SCALING["low"])).clamp(0.0, 1.0)
    return f * keep + f / SCALING["factor"] * (1.0 - keep)


SCALING = {"factor": 16.0, "context": 8192, "low": 1.0, "high": 32.0}


def _magnitude(case):
    return 0.1 * math.log(SCALING["factor"]) + 1.0 if case["scaled"] else 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"] == "rotary":
        return _prepare_rotary(case, g)
    cached, new = (torch.tensor(v, device="cuda") for v in _ragged(case))
    block = case["block"]
    if case["op"] == "blocks":
        # what is kept of a sequence: all, a little less than all (a tree of which a branch was accepted), or nothing (another request's turn)
        lens = cached + (torch.rand(case["seqs"], device="cuda", generator=g) * 24).long()
        keep = cached.clone()
        if not case["tree"]:
            keep[::3], new[1::3], new[2::3] = 0, 1, 1
            keep[1::3] = lens[1::3]
        width = -(-(case["context"] + max(24, case["new"])) // block) + 1
        blocks = int(((cached + 24 + block - 1) // block + (cached + new + 24 + block - 1) // block).sum()) + 5
        table, free, held = _table(case["seqs"], lens, block, width, blocks, g)
        total = int(new.sum())
        tokens = total + 3                              # the batch is padded
        parents = torch.cat((_parents(new, g), torch.full((3,), -1, dtype=torch.int32, device="cuda"))) if case["tree"] else None
        return {"case": case, "lens": lens.int(), "keep": keep.int(), "new": new.int(), "table": table, "free": free.contiguous(),
                "count": torch.tensor([blocks - held], dtype=torch.int32, device="cuda"), "tokens": tokens, "parents": parents}
    total = int(new.sum())
    lens = cached + new
    width = int(-(-(lens.max()) // block))
    blocks = int(((lens + block - 1) // block).sum()) + 3
    table, _, _ = _table(case["seqs"], lens, block, width, blocks, g)
    starts = torch.cat((lens.new_zeros(1), torch.cumsum(new, 0))).int()
    dt = DTYPES[case["type"]]
    if case["op"] == "move":
        caches = torch.empty((2 * case["layers"], blocks, block, case["kv"], case["dim"]), dtype=dt, device="cuda").normal_(generator=g)
        # every sequence accepts a branch: some of its new tokens, in order, a token of a branch never before its place there
        most = max(1, case["new"] // 2)
        gaps = torch.randint(1, 3, (case["seqs"], most), device="cuda", generator=g)
        kept = torch.cumsum(gaps, 1) - 1
        n_kept = (kept < new[:, None]).sum(1)
        return {"case": case, "caches": caches, "list": [c for c in caches], "table": table, "starts": starts, "lens": lens.int(), "kept": kept.int(),
                "n_kept": n_kept.int()}
    k = torch.empty((blocks, block, case["kv"], case["dim"]), dtype=dt, device="cuda").normal_(generator=g)
    v = torch.empty((blocks, block, case["kv"], case["dim"]), dtype=dt, device="cuda").normal_(generator=g)
    q = torch.empty((total, case["heads"], case["dim"]), dtype=dt, device="cuda").normal_(0.0, 2.0, generator=g)
    mask = _closure(_parents(new, g), starts, 1)[0] if case["mask"] == "tree" else None
    return {"case": case, "q": q, "k": k, "v": v, "table": table, "lens": lens.int(), "starts": starts, "mask": mask,
            "new": -(-total // case["seqs"]), "out": torch.empty_like(q), "lse": torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")}


def _prepare_rotary(case, g):
    tokens, dt, dim = case["tokens"], DTYPES[case["type"]], case["dim"]
    # queries, keys and values lie side by side, as one product leaves them
    wide = torch.randn((tokens, (case["heads"] + 2 * case["kv"]) * dim), device="cuda", generator=g).to(dt)
    q, k, v = (t.view(tokens, -1, dim) for t in wide.split([case["heads"] * dim, case["kv"] * dim, case["kv"] * dim], dim=1))
    first = int(torch.randint(0, case["far"], (1,), device="cuda", generator=g))
    positions = (first + torch.arange(tokens, device="cuda")).int()
    state = {"case": case, "q": q, "k": k, "v": v, "positions": positions, "frequencies": _frequencies(case, "cuda"),
             "q_out": torch.empty((tokens, case["heads"], dim), dtype=dt, device="cuda")}
    if case["pass"] == "cache":
        block = 16
        blocks = -(-tokens // block) + 2
        slots = torch.randperm(blocks * block, device="cuda", generator=g)[:tokens]
        if tokens > 8:
            slots[5::7] = -1                            # rows that are padding
        state["slots"] = slots
        state["caches"] = torch.zeros((2, blocks, block, case["kv"], dim), dtype=dt, device="cuda")
    else:
        state["k_out"] = torch.empty((tokens, case["kv"], dim), dtype=dt, device="cuda")
    return state


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    return {"blocks": (_blocks, _own_blocks), "rotary": (_rotary, _own_rotary), "attention": (_attention, _own_attention),
            "move": (_move, _own_move)}[state["case"]["op"]][bool(own)](state)


def _own_blocks(s):
    case = s["case"]
    starts, slots, positions, mask = context().fq_cache_step(s["lens"], s["keep"], s["new"], s["table"], s["free"], s["count"], case["block"], s["tokens"],
                                                             parents=s["parents"])
    return {"lens": s["lens"], "table": s["table"], "free": s["free"], "count": s["count"], "starts": starts, "slots": slots, "positions": positions,
            "mask": mask}


def _own_rotary(s):
    case = s["case"]
    kind = {"interleaved": case["pairs"] == "interleaved", "magnitude": _magnitude(case)}
    if case["pass"] == "cache":
        q = context().fq_rotary_cache(s["q"], s["k"], s["v"], s["positions"], s["slots"], turns(case), s["caches"][0], s["caches"][1], q_out=s["q_out"], **kind)
        return {"q": q, "caches": s["caches"]}
    q, k = context().fq_rotary(s["q"], s["k"], s["positions"], turns(case), q_out=s["q_out"], k_out=s["k_out"], inverse=case["pass"] == "gradient", **kind)
    return {"q": q, "k": k}


def _own_attention(s):
    out = context().fq_tree_attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["starts"], mask=s["mask"], out=s["out"], lse=s["lse"], new=s["new"])
    return {"out": out, "lse": s["lse"]}


def _own_move(s):
    keep = context().fq_cache_move(s["list"], s["table"], s["starts"], s["lens"], s["kept"], s["n_kept"])
    return {"caches": s["caches"], "keep": keep}


def _blocks(s):
    case, block, table, free = s["case"], s["case"]["block"], s["table"], s["free"]
    lens, keep, new = s["lens"].long(), s["keep"].long(), s["new"].long()
    have, left, want = ((n + block - 1) // block for n in (lens, keep, keep + new))
    col = torch.arange(table.shape[1], device=table.device)[None]
    room = free.shape[0]

    def places(of):                                     # exclusive sums
        return torch.cumsum(of, 0) - of

    back = have - left
    at = torch.where((col >= left[:, None]) & (col < have[:, None]), s["count"].long() + places(back)[:, None] + col - left[:, None], room)
    pool = torch.cat((free, free.new_zeros(1))).scatter(0, at.reshape(-1), table.reshape(-1))
    count = s["count"].long() + back.sum()
    taken = want - left
    at = (count - 1 - places(taken)[:, None] - (col - left[:, None])).clamp(0, room)
    grown = (col >= left[:, None]) & (col < want[:, None])
    table.copy_(torch.where(grown, pool[at.reshape(-1)].view_as(at), torch.where(col < left[:, None], table, -1)))
    free.copy_(pool[:room])
    s["count"].copy_(count - taken.sum())
    s["lens"].copy_(keep + new)
    starts = torch.cat((new.new_zeros(1), torch.cumsum(new, 0)))
    row = torch.arange(s["tokens"], device=table.device)
    seq = torch.searchsorted(starts[1:].contiguous(), row, right=True).clamp(max=case["seqs"] - 1)
    there = row < starts[-1]
    cell = keep[seq] + row - starts[seq]
    slots = torch.where(there, table[seq, (cell // block).clamp(max=table.shape[1] - 1)].long() * block + cell % block, -1)
    out = {"lens": s["lens"], "table": table, "free": free, "count": s["count"], "starts": starts.int(), "slots": slots, "mask": None}
    if s["parents"] is None:
        return {**out, "positions": torch.where(there, cell, 0).int()}
    # (padding: a tree of its own)
    bits, depth = _closure(s["parents"], torch.cat((starts, starts.new_tensor([s["tokens"]]))), 1)
    return {**out, "positions": torch.where(there, keep[seq] + depth, 0).int(), "mask": torch.where(there[:, None], bits, 0)}


def _turned(x, cos, sin, case):
    """x [tokens][heads][dim] with the pairs of its first `rot` values turned."""
    rot = case["rot"]
    y = x.float()
    if case["pairs"] == "interleaved":
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        part = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=3).reshape(*y.shape[:2], rot)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        part = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=2)
    return torch.cat((part, y[..., rot:]), dim=2).to(x.dtype)


def _rotary(s):
    case = s["case"]
    angle = s["positions"].double()[:, None] * s["frequencies"][None]
    size = _magnitude(case)
    cos, sin = ((f(angle) * size).float()[:, None] for f in (torch.cos, torch.sin))
    if case["pass"] == "gradient":
        sin = -sin
    s["q_out"].copy_(_turned(s["q"], cos, sin, case))
    k = _turned(s["k"], cos, sin, case)
    if case["pass"] != "cache":
        s["k_out"].copy_(k)
        return {"q": s["q_out"], "k": s["k_out"]}
    stored = s["slots"] >= 0
    flat = s["caches"].view(2, -1, case["kv"], case["dim"])
    flat[0, s["slots"][stored]] = k[stored]
    flat[1, s["slots"][stored]] = s["v"][stored]
    return {"q": s["q_out"], "caches": s["caches"]}


def _attention(s):
    case, q, block = s["case"], s["q"], s["case"]["block"]
    starts, lens = s["starts"].long(), s["lens"].long()
    new = starts[1:] - starts[:-1]
    most, longest, kv = case["new"], case["context"] + case["new"], case["kv"]
    i, j = torch.arange(most, device=q.device), torch.arange(longest, device=q.device)
    row = torch.where(i[None] < new[:, None], starts[:-1, None] + i[None], 0)            # [seqs][most]
    cell = s["table"].long()[:, (j // block).clamp(max=s["table"].shape[1] - 1)].clamp(min=0) * block + j % block
    keys, values = (t.view(-1, kv, case["dim"])[cell].float().transpose(1, 2) for t in (s["k"], s["v"]))       # [seqs][kv][longest][dim]
    queries = q[row].float().view(case["seqs"], most, kv, -1, case["dim"]).permute(0, 2, 3, 1, 4).flatten(2, 3)   # [seqs][kv][share * most][dim]
    scores = (queries @ keys.transpose(2, 3)).mul_(case["dim"] ** -0.5)
    nth = j[None] - (lens - new)[:, None]                                                # which new token a key is; negative: cached before
    if s["mask"] is None:
        sees = nth[:, None, :] <= i[None, :, None]
    else:
        sees = (nth[:, None, :] < 0) | ((s["mask"][row][:, :, 0:1] >> nth.clamp(0, 63)[:, None, :]) & 1).bool()
    sees &= j[None, None] < lens[:, None, None]
    view = scores.view(case["seqs"], kv, -1, most, longest)
    view.masked_fill_(~sees[:, None, None], -math.inf)
    top = scores.amax(dim=3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    scores = scores.sub_(top).exp_()
    total = scores.sum(dim=3, keepdim=True)
    some = torch.where(total > 0, total, 1.0)
    out = ((scores @ values) / some).view(case["seqs"], kv, -1, most, case["dim"]).permute(0, 3, 1, 2, 4).reshape(case["seqs"], most, case["heads"], -1)
    lse = (torch.log(total) + top)[..., 0].view(case["seqs"], kv, -1, most).permute(0, 3, 1, 2).reshape(case["seqs"], most, case["heads"])
    real = torch.repeat_interleave(torch.arange(case["seqs"], device=q.device), new, output_size=q.shape[0])
    nth_row = torch.arange(q.shape[0], device=q.device) - starts[real]
    s["out"].copy_(out[real, nth_row])
    s["lse"].copy_(lse[real, nth_row])
    return {"out": s["out"], "lse": s["lse"]}


def _move(s):
    case, block = s["case"], s["case"]["block"]
    starts, lens, kept = s["starts"].long(), s["lens"].long(), s["kept"].long()
    before = lens - (starts[1:] - starts[:-1])
    i = torch.arange(kept.shape[1], device=kept.device)[None]
    asked = (i < s["n_kept"][:, None]) & (kept != i)

    def slots(cell):
        return torch.gather(s["table"].long(), 1, (cell // block).clamp(max=s["table"].shape[1] - 1)) * block + cell % block

    source, target = slots(before[:, None] + kept)[asked], slots(before[:, None] + i)[asked]
    flat = s["caches"].view(2 * case["layers"], -1, case["kv"], case["dim"])
    flat[:, target] = flat[:, source]
    return {"caches": s["caches"], "keep": (before + s["n_kept"]).int()}


# ---------------------------------------------------------------------------------------------------------------- reckoning
def work(case):
    if case["op"] == "rotary":
        tokens, e = case["tokens"], SIZE[case["type"]]
        elements = tokens * (case["heads"] + (2 if case["pass"] == "cache" else 1) * case["kv"]) * case["dim"]
        return {"bytes": 2 * elements * e + tokens * 12, "flops": 3 * elements}
    cached, new = _ragged(case)
    if case["op"] == "blocks":
        if not case["tree"]:
            new = [n if b % 3 == 0 else 1 for b, n in enumerate(new)]
        blocks = sum(-(-n // case["block"]) + 1 for n in new)
        return {"bytes": 16 * case["seqs"] + 16 * blocks + sum(new) * (24 if case["tree"] else 12), "flops": 0}
    e = SIZE[case["type"]]
    if case["op"] == "move":
        moved = sum(n // 2 for n in new)
        return {"bytes": 4 * case["layers"] * moved * case["kv"] * case["dim"] * e, "flops": 0}
    rows, keys = sum(new), sum(c + n for c, n in zip(cached, new) if n)
    pairs = sum(n * c + n * (n + 1) / 2 for c, n in zip(cached, new))
    return {"bytes": 2 * keys * case["kv"] * case["dim"] * e + 2 * rows * case["heads"] * case["dim"] * e + 4 * rows * case["heads"],
            "flops": 4 * pairs * case["heads"] * case["dim"]}


def exact(case, seed):
    """From the definitions, in 64 bits, a sequence at a time."""
    if case["op"] in ("blocks", "move"):
        return None                                      # whole numbers, and values that are only copied
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_rotary(case, s)
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    share = case["heads"] // case["kv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        n, length = starts[b + 1] - starts[b], lens[b]
        if n == 0:
            continue
        cells = s["table"][b, torch.arange(length, device="cuda") // case["block"]].long(), torch.arange(length, device="cuda") % case["block"]
        allowed = torch.ones((n, length), dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            allowed = allowed.tril(length - n)
        else:
            bits = s["mask"][starts[b]:starts[b + 1], 0]
            allowed[:, length - n:] = torch.stack([(bits >> t) % 2 == 1 for t in range(n)], dim=1)
        for h in range(case["kv"]):
            key, value = s["k"][cells[0], cells[1], h].double(), s["v"][cells[0], cells[1], h].double()
            for r in range(h * share, (h + 1) * share):
                z = s["q"][starts[b]:starts[b + 1], r].double() @ key.T / math.sqrt(case["dim"])
                z = z.masked_fill(~allowed, -math.inf)
                lse[starts[b]:starts[b + 1], r] = torch.logsumexp(z, 1)
                out[starts[b]:starts[b + 1], r] = torch.softmax(z, 1) @ value
    return {"out": out, "lse": lse}


def _exact_rotary(case, s):
    """Pairs as complex numbers, multiplied with magnitude * exp(i angle)."""
    pairs = case["rot"] // 2
    rate = torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)], dtype=torch.float64)
    if case["scaled"]:
        weight = ((SCALING["context"] * rate / math.tau - SCALING["low"]) / (SCALING["high"] - SCALING["low"])).clamp(0, 1)
        rate = rate * (weight + (1 - weight) / SCALING["factor"])
    angle = torch.outer(s["positions"].double(), rate.cuda()) * (-1 if case["pass"] == "gradient" else 1)
    spin = torch.polar(torch.full_like(angle, _magnitude(case)), angle).unsqueeze(1)

    def turned(x):
        x = x.double().clone()
        first, second = (slice(0, case["rot"], 2), slice(1, case["rot"], 2)) if case["pairs"] == "interleaved" else (slice(0, pairs), slice(pairs, 2 * pairs))
        z = torch.complex(x[..., first], x[..., second]) * spin
        x[..., first], x[..., second] = z.real, z.imag
        return x

    if case["pass"] != "cache":
        return {"q": turned(s["q"]), "k": turned(s["k"])}
    caches = s["caches"].double()
    key, slots = turned(s["k"]), s["slots"].tolist()
    rows = torch.tensor([t for t, c in enumerate(slots) if c >= 0], device="cuda")
    caches.view(2, -1, case["kv"], case["dim"])[0, s["slots"][rows]] = key[rows]
    caches.view(2, -1, case["kv"], case["dim"])[1, s["slots"][rows]] = s["v"][rows].double()
    return {"q": turned(s["q"]), "caches": caches}
