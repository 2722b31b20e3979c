"""Cache tables, rotary positions, attention and moves together: a block's attention in the search, and steps of drafting and verifying a tree."""
import math
from collections import namedtuple

import pytest
import torch

import fq_paged as O
from fq_testlib import make_layer, to_dev, x_bf16

pytestmark = pytest.mark.gpu
Shape = namedtuple("Shape", "n_out k_in")


def turned(x, positions, base=10000.0):
    """Rotary positions in 64 bits, the two halves of a head paired."""
    half = x.shape[-1] // 2
    angle = positions.double().cuda()[:, None] * torch.tensor([base ** (-i / half) for i in range(half)], dtype=torch.float64, device="cuda")
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x.double()[..., :half], x.double()[..., half:]
    return torch.cat((a * c - b * s, a * s + b * c), 2)


def causal(q, k, v, lengths):
    """Attention of sequences on their own, in 64 bits."""
    out, at, share = [], 0, q.shape[1] // k.shape[1]
    for n in lengths:
        z = torch.einsum("nhd,lhd->hnl", q[at:at + n], k[at:at + n].repeat_interleave(share, 1)) / math.sqrt(q.shape[2])
        z = z.masked_fill(~torch.ones((n, n), dtype=torch.bool, device="cuda").tril(), -math.inf)
        out.append(torch.einsum("hnl,lhd->nhd", torch.softmax(z, 2), v[at:at + n].repeat_interleave(share, 1)))
        at += n
    return torch.cat(out)


@pytest.mark.parametrize("heads,kv,dim,lengths", [(4, 4, 64, (30, 1, 17)), (8, 2, 32, (48,)), (16, 1, 16, (40, 8))])
def test_attention_in_an_ensemble(heads, kv, dim, lengths):
    import paper_2501_07139_b200 as P
    from paper_2501_07139_b200 import search as SR
    hidden, levels, tokens, sens = 256, [8, 5, 3], 48, 16
    shapes = [Shape(heads * dim, hidden), Shape(kv * dim, hidden), Shape(kv * dim, hidden), Shape(hidden, heads * dim), Shape(96, hidden)]
    fq = P.FlexQ(5)
    for i, sh in enumerate(shapes):
        fq.fq_pack_layer(i, *to_dev(*make_layer(180, i, sh.n_out, sh.k_in, 8)), 8, P.FQ_FMT_PLANES)
    x = x_bf16(180, hidden, tokens, hidden).cuda() * 4
    att = SR.Attention(0, 1, 2, 3, heads, kv, lengths, block_size=16)
    calib = {256: x}
    if heads * dim != hidden:
        calib[heads * dim] = x_bf16(180, heads * dim, tokens, heads * dim).cuda()
    modules = [[0, 1, 2, 3], [4]]
    plain = SR.module_tables(fq, shapes, modules, levels, calib, sens)
    out = SR.generate_ensemble(fq, shapes, modules, levels, calib, sens_tokens=sens, attention=[att])
    assert out["cost"][1] == plain[0][1] and out["sens"][1] == plain[1][1] and out["foot"] == plain[2]       # the others are evaluated as before
    # references from the library's own products, in 64 bits between them
    ys, refs = [], []
    for b in levels:
        fq.fq_set_config([b, b, b, b, 8])
        ys.append(SR.attention_outputs(fq, att, shapes, x))
        q, k, v = (fq.fq_gemm(i, x, SR._outputs(tokens, shapes[i].n_out, x.device)).view(tokens, -1, dim) for i in (0, 1, 2))
        pos = torch.cat([torch.arange(n) for n in lengths])
        q, k = (turned(t, pos).bfloat16().double() for t in (q, k))
        ref = causal(q, k, v.double(), lengths).bfloat16().reshape(tokens, heads * dim)
        refs.append(fq.fq_gemm(3, ref, SR._outputs(tokens, hidden, x.device)))
        # a few roundings of 2^-8 between the two, averaged by the products: relative L2
        err = float((ys[-1].double() - refs[-1].double()).norm() / refs[-1].double().norm())
        assert err <= 3 * 2.0 ** -8, (b, err)
    for li in range(3):
        for rows, table in ((slice(None), "cost"), (slice(sens), "sens")):
            d = (ys[li][rows].double() - ys[0][rows].double()).square().sum() / ys[0][rows].double().square().sum()
            assert abs(out[table][0][li] - float(d)) <= 1e-9 * max(1.0, float(d))
    assert out["cost"][0][0] == 0.0 and 0.0 < out["cost"][0][1] < out["cost"][0][2]
    for bad in (att._replace(o=4), att._replace(lengths=(5,)), att._replace(kv_heads=kv * 2)):
        with pytest.raises(ValueError):
            SR.module_tables(fq, shapes, modules, levels, calib, sens, attention=[bad])
    assert fq.fq_status() == 0
    fq.fq_destroy()


@pytest.mark.parametrize("dt,heads,kv,dim,block", [(torch.float16, 4, 4, 128, 16), (torch.bfloat16, 8, 2, 64, 5)])
def test_drafting_and_verifying(dt, heads, kv, dim, block):
    """Two sequences: a prompt, then trees of drafted tokens of which a branch is kept, over two layers' caches.  What a token finds in the end is what it
    would have found had the kept tokens come one by one."""
    import paper_2501_07139_b200 as P
    fq, layers, n = P.FlexQ(1), 2, 2
    g = torch.Generator().manual_seed(7)
    gd = torch.Generator(device="cuda").manual_seed(7)
    width, blocks = 80 // block + 1, 2 * (80 // block + 1)
    d = dict(lens=torch.zeros(n, dtype=torch.int32, device="cuda"), table=torch.full((n, width), -1, dtype=torch.int32, device="cuda"),
             free=torch.randperm(blocks, generator=g).int().cuda(), count=torch.tensor([blocks], dtype=torch.int32, device="cuda"))
    caches = [torch.full((2, blocks, block, kv, dim), math.nan, dtype=dt, device="cuda") for _ in range(layers)]
    turns = P.fq_rotary_table(dim)
    keep = torch.zeros(n, dtype=torch.int32, device="cuda")
    history = [[] for _ in range(n)]             # of every sequence: what was kept, (q, k, v) of each layer

    def step(new, parents):
        total = sum(new)
        qkv = [[torch.randn((total, h, dim), device="cuda", generator=gd).to(dt) for h in (heads, kv, kv)] for _ in range(layers)]
        starts, slots, positions, mask = fq.fq_cache_step(d["lens"], keep, torch.tensor(new, dtype=torch.int32, device="cuda"), d["table"], d["free"],
                                                          d["count"], block, total + 2, parents=parents)
        outs = []
        for (q, k, v), c in zip(qkv, caches):
            pad = [torch.cat((t, t.new_zeros((2, *t.shape[1:])))) for t in (q, k, v)]          # the batch is padded
            rq = fq.fq_rotary_cache(*pad, positions, slots, turns, c[0], c[1])
            outs.append(fq.fq_tree_attention(rq, c[0], c[1], d["table"], d["lens"], starts, mask=mask)[:total])
        return qkv, outs, starts

    def reference(b, branch_qkv, layer):
        """The last token of a sequence whose tokens are the kept ones and those of the branch, in 64 bits."""
        q, k, v = (torch.cat([t[layer][i][None] for t in history[b] + branch_qkv]) for i in range(3))
        pos = torch.arange(q.shape[0])
        q, k = (turned(t, pos).to(dt).double() for t in (q, k))
        return causal(q, k, v.double(), [q.shape[0]])[-1]

    qkv, outs, _ = step([9, 14], None)
    for b, rows in enumerate((range(9), range(9, 23))):
        history[b] = [[[t[i] for t in qkv[layer]] for layer in range(layers)] for i in rows]
    keep = torch.tensor([9, 14], dtype=torch.int32, device="cuda")
    for turn in range(4):
        new = [6, 3 + turn]
        trees = [O.tree(v, g) for v in new]
        qkv, outs, starts = step(new, torch.tensor(sum(trees, []) + [-1, -1], dtype=torch.int32, device="cuda"))
        branches = []
        for b in range(n):
            first = sum(new[:b])
            token = [[[t[first + i] for t in qkv[layer]] for layer in range(layers)] for i in range(new[b])]
            ways = []
            for i in range(new[b]):
                way, p = [i], trees[b][i]
                while p >= 0:
                    way.insert(0, p)
                    p = trees[b][p]
                ways.append(way)
                for layer in range(layers):
                    want = reference(b, [token[j] for j in way], layer)
                    # weights and results are rounded by half a step each; values are a few
                    step_of = 2.0 ** -11 if dt == torch.float16 else 2.0 ** -8
                    assert float((outs[layer][first + i].double() - want).abs().max()) <= 2 * 4.5 * step_of
            chosen = ways[int(torch.randint(0, new[b], (1,), generator=g))] if turn != 2 else []
            branches.append(chosen)
            history[b] += [token[j] for j in chosen]
        most = max(1, max(map(len, branches)))
        kept = torch.tensor([w + [0] * (most - len(w)) for w in branches], dtype=torch.int32, device="cuda")
        keep = fq.fq_cache_move([c[i] for c in caches for i in range(2)], d["table"], starts, d["lens"], kept,
                                torch.tensor([len(w) for w in branches], dtype=torch.int32, device="cuda"))
        assert keep.tolist() == [len(h) for h in history]
    held = [x for r in d["table"].tolist() for x in r if x >= 0] + d["free"].tolist()[:int(d["count"])]
    assert sorted(held) == list(range(blocks)) and fq.fq_status() == 0
    fq.fq_destroy()
