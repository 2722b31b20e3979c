"""Attention of new tokens over paged caches against the definition in 64 bits."""
import math

import pytest
import torch

import fq_paged as O

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    c.fq_destroy()


def dev(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def make(ctx, new, heads, kv, dim, block, dt, tree=False, seed=1, pad=0, heads_first=False, words=None, spare=2):
    """Caches full of NaN but for the sequences' cells."""
    g = torch.Generator().manual_seed(seed)
    lens = [a + b for a, b in zip(ctx, new)]
    width = max(1, max(O.ceil_div(v, block) for v in lens))
    blocks = sum(O.ceil_div(v, block) for v in lens) + spare
    table, _ = O.make_table(lens, block, width, blocks, g)
    shape = (blocks, kv, block, dim) if heads_first else (blocks, block, kv, dim)
    k, v = (torch.full(shape, math.nan, dtype=dt, device="cuda") for _ in range(2))
    if heads_first:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    gd = torch.Generator(device="cuda").manual_seed(seed)
    table = table.cuda()
    for b, n in enumerate(lens):
        cells = torch.arange(n, device="cuda")
        at = table[b].long()[cells // block], cells % block
        k[at], v[at] = (torch.randn((n, kv, dim), device="cuda", generator=gd).to(dt) for _ in range(2))
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    tokens = max(1, starts[-1] + pad)
    q = (torch.randn((tokens, heads, dim), device="cuda", generator=gd) * 1.5).to(dt)
    mask = None
    if tree:
        words = words or max(1, O.ceil_div(max(new), 64))
        mask = [row for n in new for row in O.tree_bits(O.tree(n, g), words)] + [[-1] * words] * (tokens - starts[-1])
        mask = dev(mask, torch.int64)
    return dict(q=q, k=k, v=v, table=table, lens=lens, starts=starts, mask=mask)


def call(fq, s, **more):
    out = torch.full(s["q"].shape, 77.0, dtype=s["q"].dtype, device="cuda")
    lse = torch.full(s["q"].shape[:2], 77.0, device="cuda")
    args = dict(out=out, lse=lse, mask=s["mask"])
    args.update(more)
    got = fq.fq_tree_attention(s["q"], s["k"], s["v"], s["table"], dev(s["lens"]), dev(s["starts"]), **args)
    assert got is args["out"]
    return got, args["lse"]


def check(s, out, lse, scale=None, only=None):
    """Every element: half a step of the result; half a step of each weight (times sum p |v|), of subnormal fp16 weights 2^-25 each; scores, exponentials and sums
    in fp32: dim + 8 roundings of sum |q k|, 2^-21 for an exponential, n + 64 of 2^-24 for sums of n weights."""
    want, want_lse = O.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["starts"], s["mask"], scale)
    heads, dim = s["q"].shape[1:]
    scale = dim ** -0.5 if scale is None else scale
    h, block = HALF_STEP[out.dtype], s["k"].shape[1]
    for b, n in enumerate(s["lens"]):
        rows = slice(s["starts"][b], s["starts"][b + 1])
        if rows.start == rows.stop or (only is not None and b not in only):
            continue
        cells = torch.arange(n, device="cuda")
        at = s["table"][b].long()[cells // block] if n else cells, cells % block
        most_v = s["v"][at].double().abs().nan_to_num(0, 0).amax() if n else 0.0
        size = s["q"][rows].double().abs().amax() * s["k"][at].double().abs().nan_to_num(0, 0).amax() * dim * scale if n else 0.0
        d = (dim + 8) * 2.0 ** -24 * size + 2.0 ** -21 + (n + 64) * 2.0 ** -24
        w = want[rows]
        bound = w.abs() * h + most_v * (h + 2 * d + (n * 2.0 ** -25 if out.dtype == torch.float16 else 0.0))
        fine = w.isfinite()
        assert torch.equal(fine, out[rows].isfinite())
        assert bool(((out[rows].double() - w).abs() <= bound)[fine].all()), (b, float(((out[rows].double() - w).abs() - bound)[fine].max()))
        e = want_lse[rows]
        assert torch.equal(e == -math.inf, lse[rows] == -math.inf) and torch.equal(e.isnan(), lse[rows].isnan())
        some = e.isfinite()
        assert bool(((lse[rows].double() - e).abs() <= d + e.abs() * 2.0 ** -22)[some].all())
    end = s["starts"][-1] if only is None else len(out)
    assert bool((out[end:] == 77).all()) and bool((lse[end:] == 77).all())


# (context, new) of each sequence
LENGTHS = {
    "one": [(0, 1)], "ends": [(14, 1), (15, 1), (16, 1), (126, 1), (127, 1), (128, 1), (300, 1)], "long": [(5000, 1)], "ragged": [(900, 1), (0, 1), (3, 0), (70, 1), (0, 0), (2500, 1)],
    "drafts": [(100, 8), (0, 5), (33, 3), (1000, 7)], "prompt": [(0, 300)], "prompts": [(0, 70), (200, 33), (513, 130)], "none": [(10, 0), (0, 0)],
}


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("heads,kv,dim,block,tree", [(4, 4, 128, 16, False), (8, 2, 64, 32, True), (7, 1, 128, 5, True), (6, 3, 256, 64, False), (2, 2, 80, 1, True), (32, 4, 128, 100, True), (3, 3, 8, 16, False),
                                                     (5, 5, 160, 24, True)])
def test_attention(fq, dt, lengths, heads, kv, dim, block, tree):
    ctx, new = zip(*LENGTHS[lengths])
    s = make(ctx, new, heads, kv, dim, block, dt, tree, pad=3, heads_first=heads == 6)
    out, lse = call(fq, s)
    check(s, out, lse)
    again, lse2 = call(fq, s)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    # the number of new tokens is a hint
    for hint in (1, 4, 2048):
        other, lse3 = call(fq, s, new=hint)
        check(s, other, lse3)
    assert fq.fq_status() == 0


@pytest.mark.parametrize("ctx,new,heads,kv,words", [([64, 0, 7], [60, 64, 17], 64, 8, 1), ([1000], [200], 8, 8, 4), ([0, 20], [1000, 3], 2, 1, 16), ([5000, 17], [64, 63], 16, 2, 1)])
def test_larger_trees(fq, ctx, new, heads, kv, words):
    s = make(ctx, new, heads, kv, 128, 16, torch.bfloat16, True, words=words)
    check(s, *call(fq, s))
    assert fq.fq_status() == 0


def test_many_sequences(fq):
    g = torch.Generator().manual_seed(2)
    n = 700
    ctx, new = torch.randint(0, 90, (n,), generator=g).tolist(), torch.randint(0, 4, (n,), generator=g).tolist()
    s = make(ctx, new, 4, 2, 64, 16, torch.float16, True)
    for hint in (1, 40, 500):
        check(s, *call(fq, s, new=hint))
    assert fq.fq_status() == 0


@pytest.mark.parametrize("heads,kv,new", [(200, 1, 3), (96, 2, 5), (128, 1, 2), (24, 8, 100)])
def test_large_and_odd_groups(fq, heads, kv, new):
    """Query heads to a key head: more than a tile of rows, sizes that do not divide it."""
    s = make([150, 0], [new, new], heads, kv, 64, 16, torch.bfloat16, True, words=2)
    for hint in (1, 40, 500):
        check(s, *call(fq, s, new=hint))
    assert fq.fq_status() == 0


def test_queries_that_are_repeated(fq):
    """One token's queries, or one head's, for all: strides of 0."""
    s = make([100, 30], [20, 33], 8, 2, 128, 16, torch.float16)
    for q in (s["q"][:1].expand(53, 8, 128), s["q"][:, :1].expand(53, 8, 128)):
        want, lse = call(fq, {**s, "q": q.contiguous()})
        for hint in (1, 20, 500):
            got, lse2 = call(fq, {**s, "q": q}, new=hint)
            check({**s, "q": q.contiguous()}, got, lse2)
            same, lse3 = call(fq, {**s, "q": q.contiguous()}, new=hint)
            assert torch.equal(got, same) and torch.equal(lse2, lse3)
    assert fq.fq_status() == 0


@pytest.mark.parametrize("heads,kv", [(4, 4), (16, 2), (64, 2)])
def test_rows_that_see_nothing(fq, heads, kv):
    """Bits that leave a row empty, with nothing cached before; bits beyond the new tokens; rows that see one."""
    s = make([0, 0, 40], [5, 70, 3], heads, kv, 128, 16, torch.bfloat16, True, words=2)
    m = s["mask"]
    m[0], m[2] = 0, 0
    m[3] = -1                                       # all five, and what is not there
    m[5 + 7], m[5 + 69] = 0, 0
    m[75] = 0                                       # sees what is cached
    out, lse = call(fq, s)
    check(s, out, lse)
    assert not bool(out[[0, 2, 12, 74]].any()) and bool((lse[[0, 2, 12, 74]] == -math.inf).all())
    assert fq.fq_status() == 0


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 128), (16, 2, 64), (64, 2, 128), (4, 1, 256)])
@pytest.mark.parametrize("tree", [False, True])
def test_what_is_not_seen_does_not_touch(fq, dt, heads, kv, dim, tree):
    """Infinities and NaNs in keys and values of new tokens: rows that see the token are spoilt, all others are what they would be without."""
    s = make([50, 0, 130], [9, 40, 70], heads, kv, dim, 16, dt, tree, words=2)
    clean, lse0 = call(fq, s)
    block = 16

    def place(b, nth):
        cell = s["lens"][b] - (s["starts"][b + 1] - s["starts"][b]) + nth
        return int(s["table"][b, cell // block]), cell % block

    hit = [(0, 4, "v", math.nan), (0, 6, "v", math.inf), (1, 33, "v", -math.inf), (1, 20, "k", math.nan), (2, 66, "k", math.inf), (2, 50, "v", math.nan)]
    for b, nth, which, value in hit:
        at = place(b, nth)
        s[which][at[0], at[1], kv - 1, 3] = value
    out, lse = call(fq, s)
    spoilt = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    share = heads // kv
    for b, nth, which, _ in hit:
        for i in range(s["starts"][b + 1] - s["starts"][b]):
            row = s["starts"][b] + i
            seen = bool(int(s["mask"][row, nth // 64]) >> (nth % 64) & 1) if tree else nth <= i
            if seen:
                if which == "v":
                    spoilt[row, (kv - 1) * share:, 3] = True
                else:
                    spoilt[row, (kv - 1) * share:] = True
    assert torch.equal(out[~spoilt], clean[~spoilt])
    only_v = spoilt.clone()
    for b, nth, which, _ in hit:
        if which == "k":
            for i in range(s["starts"][b + 1] - s["starts"][b]):
                row = s["starts"][b] + i
                if bool(int(s["mask"][row, nth // 64]) >> (nth % 64) & 1) if tree else nth <= i:
                    only_v[row] = False
    assert not bool(out[only_v].isfinite().any())
    assert bool(spoilt.any()) and fq.fq_status() == 0


def test_large_scores(fq):
    """Scores up to some hundreds: the largest decides, and none overflows."""
    s = make([333, 90], [2, 1], 4, 2, 128, 16, torch.bfloat16)
    s["q"] *= 40
    check(s, *call(fq, s))
    s["q"][0] = 0                                   # all weights alike
    check(s, *call(fq, s))
    check(s, *call(fq, s, scale=1e-3), scale=1e-3)
    assert fq.fq_status() == 0


@pytest.mark.parametrize("new,heads", [(1, 4), (5, 4), (70, 16)])
def test_strides(fq, new, heads):
    """Queries as a part of a wider buffer, outputs with heads first, a table inside a wider one."""
    dim, kv = 64, 2
    s = make([100, 3], [new, new], heads, kv, dim, 16, torch.float16)
    want, lse = call(fq, s)
    wide = torch.randn((2 * new, heads + 4, dim + 8), device="cuda").half()
    part = wide[:, 2:2 + heads, 8:]
    part.copy_(s["q"])
    out = torch.full((heads, 2 * new, dim), 77.0, device="cuda").half().transpose(0, 1)
    table = torch.full((2, s["table"].shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    table[:, :s["table"].shape[1]] = s["table"]
    got, lse2 = call(fq, {**s, "q": part, "table": table[:, :s["table"].shape[1] + 1]}, out=out)
    assert torch.equal(got, want) and torch.equal(lse, lse2) and fq.fq_status() == 0


@pytest.mark.parametrize("new,heads", [(1, 4), (70, 16)])
def test_numbers_that_cannot_be(fq, new, heads):
    s = make([100, 30, 60], [new, new, new], heads, 2, 128, 16, torch.bfloat16, spare=0)
    call(fq, s)
    blocks = s["k"].shape[0]
    # blocks that are not there count as zeros; the other sequences do not notice
    bad = dict(s, table=s["table"].clone())
    bad["table"][1, 0], bad["table"][1, 1] = blocks, -5
    got, _ = call(fq, bad)
    assert fq.fq_status() == -14
    zeroed = dict(s, k=s["k"].clone(), v=s["v"].clone())
    for j in (0, 1):
        zeroed["k"][int(s["table"][1, j])], zeroed["v"][int(s["table"][1, j])] = 0, 0
    ref, _ = call(fq, zeroed)
    assert torch.equal(got, ref)
    # fewer cells than new tokens: its rows see nothing.  (The others' work is dealt in another way: their last bits may differ.)
    got, lse = call(fq, dict(s, lens=[s["lens"][0], new - 1, s["lens"][2]]))
    assert fq.fq_status() == -14 and not bool(got[new:2 * new].any()) and bool((lse[new:2 * new] == -math.inf).all())
    check(s, got, lse, only=(0, 2))
    # lengths beyond the table, rows beyond the batch
    got, lse = call(fq, dict(s, lens=[s["lens"][0], 2**31 - 1, s["lens"][2]]))
    assert fq.fq_status() == -14
    check(s, got, lse, only=(0, 2))
    got, lse = call(fq, dict(s, starts=[0, new, 2 * new, 2**31 - 1]))
    assert fq.fq_status() == -14 and bool((got[2 * new:] == 77).all())
    check(s, got, lse, only=(0, 1))
    got, lse = call(fq, dict(s, starts=[0, new, -3, -2**31]))
    assert fq.fq_status() == -14 and bool((got[new:] == 77).all())
    check(s, got, lse, only=(0,))
    assert fq.fq_status() == 0


@pytest.mark.parametrize("new,heads", [(1, 8), (6, 8), (60, 16)])
def test_replays_see_new_lengths(fq, new, heads):
    """A captured call, replayed for other lengths; on a stream of its own, its first launch captured."""
    a, b = make([700, 40], [new, new], heads, 2, 128, 16, torch.bfloat16, seed=1), make([90, 600], [new, new], heads, 2, 128, 16, torch.bfloat16, seed=2)
    width = max(a["table"].shape[1], b["table"].shape[1])
    blocks = max(a["k"].shape[0], b["k"].shape[0])
    q, table, lens, starts = torch.empty_like(a["q"]), torch.full((2, width), -1, dtype=torch.int32, device="cuda"), dev([0, 0]), dev(a["starts"])
    k, v = (torch.zeros((blocks, *a["k"].shape[1:]), dtype=a["k"].dtype, device="cuda") for _ in range(2))
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")

    def load(s):
        q.copy_(s["q"])
        table[:, :s["table"].shape[1]] = s["table"]
        lens.copy_(dev(s["lens"]))
        k[:s["k"].shape[0]], v[:s["v"].shape[0]] = s["k"], s["v"]

    load(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fq.fq_tree_attention(q, k, v, table, lens, starts, out=out, lse=lse)
    for s in (a, b, a):
        load(s)
        graph.replay()
        torch.cuda.synchronize()
        check(s, out, lse)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            other = fq.fq_tree_attention(q, k, v, table, lens, starts)
        stream.synchronize()
        assert torch.equal(other, out)
    assert fq.fq_status() == 0
