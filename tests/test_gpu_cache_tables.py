"""Block tables, slots, positions and tree bits built on the GPU, and the move of accepted branches, against plain Python."""
import pytest
import torch

import fq_paged as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    c.fq_destroy()


def dev(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def case(n, block, longest, most, seed, trees):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, longest + 1, (n,), generator=g).tolist()
    keep = [int(torch.randint(0, v + 1, (1,), generator=g)) if i % 3 else (v if i % 2 else 0) for i, v in enumerate(lens)]
    new = torch.randint(0, most + 1, (n,), generator=g).tolist()
    width = O.ceil_div(longest + most, block) + 2
    blocks = sum(O.ceil_div(v, block) for v in lens) + sum(O.ceil_div(a + b, block) for a, b in zip(keep, new)) + 3
    table, rest = O.make_table(lens, block, width, blocks, g)
    parents = [p for v in new for p in O.tree(v, g)] if trees else None
    return lens, keep, new, table, rest, blocks, parents


@pytest.mark.parametrize("n,block,longest,most,pad,words", [(1, 16, 40, 1, 0, 0), (1, 1, 3, 5, 1, 1), (3, 16, 100, 20, 5, 1), (65, 100, 5000, 3, 0, 0), (64, 7, 60, 64, 9, 1),
                                                            (600, 32, 500, 40, 3, 2), (1100, 16, 30, 8, 0, 1), (5, 64, 300, 700, 17, 16), (17, 65536, 70000, 9, 0, 1),
                                                            (4200, 8, 20, 2, 0, 0), (2, 16, 0, 0, 4, 0)])
def test_step(fq, n, block, longest, most, pad, words):
    lens, keep, new, table, rest, blocks, parents = case(n, block, longest, most, n + block, words > 0)
    tokens = sum(new) + pad
    if tokens == 0:
        tokens = 1
    count = len(rest)
    free = rest + [-7] * (blocks - count)
    if parents is not None:
        parents = parents + [-1] * (tokens - len(parents))
    d = dict(lens=dev(lens), keep=dev(keep), new=dev(new), table=torch.full((n, table.shape[1] + 3), -9, dtype=torch.int32, device="cuda")[:, :table.shape[1]],
             free=dev(free), count=dev([count]))
    d["table"].copy_(table)
    got = fq.fq_cache_step(*d.values(), block, tokens, parents=None if parents is None else dev(parents), words=max(words, 1))
    rows = table.tolist()
    starts, slots, positions, bits, count = O.step(lens, keep, new, rows, free, count, block, tokens, parents, max(words, 1))
    assert fq.fq_status() == 0
    assert d["lens"].tolist() == lens and d["table"].tolist() == rows and d["free"].tolist() == free and d["count"].tolist() == [count]
    assert got[0].tolist() == starts and got[1].tolist() == slots and got[2].tolist() == positions
    assert got[3] is None if parents is None else got[3].tolist() == O.signed(bits)
    # what lies beside the table's rows stays
    assert n == 1 or bool((d["table"].as_strided((n - 1, 3), (table.shape[1] + 3, 1), table.shape[1]) == -9).all())


def test_a_run_of_steps(fq):
    """Requests come, draft, are cut back and leave; no block is lost or held twice."""
    g = torch.Generator().manual_seed(5)
    n, block, width, blocks = 9, 8, 12, 70
    lens, rows, free, count = [0] * n, [[-1] * width for _ in range(n)], list(range(blocks)), blocks
    d = dict(lens=dev(lens), table=dev(rows), free=dev(free), count=dev([count]))
    for turn in range(12):
        keep = [int(torch.randint(0, v + 1, (1,), generator=g)) if (turn + b) % 4 else 0 for b, v in enumerate(lens)]
        new = torch.randint(0, 12, (n,), generator=g).tolist()
        new = [min(v, width * block - k) for v, k in zip(new, keep)]
        while sum(O.ceil_div(a + b, block) for a, b in zip(keep, new)) > blocks:
            new = [v // 2 for v in new]
            keep = [v // 2 for v in keep]
        tokens = sum(new) + 2
        got = fq.fq_cache_step(d["lens"], dev(keep), dev(new), d["table"], d["free"], d["count"], block, tokens)
        starts, slots, positions, _, count = O.step(lens, keep, new, rows, free, count, block, tokens)
        assert got[0].tolist() == starts and got[1].tolist() == slots and got[2].tolist() == positions
        assert d["lens"].tolist() == lens and d["table"].tolist() == rows and d["count"].tolist() == [count] and d["free"].tolist()[:count] == free[:count]
        held = [x for r in rows for x in r if x >= 0] + free[:count]
        assert sorted(held) == list(range(blocks))
    assert fq.fq_status() == 0


@pytest.mark.parametrize("n,tokens", [(3, 40), (400, 9000)])
def test_all_go_on(fq, n, tokens):
    """The lengths themselves as what is kept."""
    g = torch.Generator().manual_seed(n)
    lens, new = torch.randint(0, 50, (n,), generator=g).tolist(), torch.randint(0, tokens // n, (n,), generator=g).tolist()
    blocks = sum(O.ceil_div(a + b, 8) for a, b in zip(lens, new)) + 2
    table, rest = O.make_table(lens, 8, 30, blocks, g)
    free, rows, count = rest + [0] * (blocks - len(rest)), table.tolist(), len(rest)
    d, t, f, c = dev(lens), table.cuda(), dev(free), dev([count])
    got = fq.fq_cache_step(d, d, dev(new), t, f, c, 8, tokens)
    starts, slots, positions, _, count = O.step(lens, list(lens), new, rows, free, count, 8, tokens)
    assert fq.fq_status() == 0 and d.tolist() == lens and t.tolist() == rows and c.tolist() == [count]
    assert got[0].tolist() == starts and got[1].tolist() == slots and got[2].tolist() == positions


BAD = {
    "blocks": (dict(count=[1]), -13), "width": (dict(new=[3, 200, 0]), -13), "rows": (dict(new=[30, 30, 30]), -13), "keep": (dict(keep=[3, 41, 0]), -14),
    "negative new": (dict(new=[1, -1, 1]), -14), "negative length": (dict(lens=[-1, 40, 5]), -14), "long": (dict(lens=[3, 4000, 5]), -14),
    "count": (dict(count=[99]), -14), "negative count": (dict(count=[-2]), -14), "huge": (dict(new=[2**31 - 1] * 3), -13),
}


@pytest.mark.parametrize("name", list(BAD))
@pytest.mark.parametrize("trees", [False, True])
def test_what_does_not_fit_changes_nothing(fq, name, trees):
    change, code = BAD[name]
    block, width, tokens = 8, 8, 64
    v = dict(lens=[3, 40, 5], keep=[3, 40, 0], new=[9, 2, 30], count=[20])
    v.update(change)
    table = torch.full((3, width), -1, dtype=torch.int32)
    for b, n in enumerate((1, 5, 1)):
        table[b, :n] = torch.arange(n) + 10 * b
    free = list(range(40, 66))
    d = {k: dev(x) for k, x in v.items()}
    t, f = table.cuda(), dev(free)
    got = fq.fq_cache_step(d["lens"], d["keep"], d["new"], t, f, d["count"], block, tokens, parents=dev([-1] * tokens) if trees else None)
    status = fq.fq_status()
    if trees and name in ("width", "huge"):
        code = -14                       # (more than a row of bits holds)
    assert status == code
    assert d["lens"].tolist() == v["lens"] and d["count"].tolist() == v["count"] and t.tolist() == table.tolist() and f.tolist() == free
    assert got[0].tolist() == [0] * 4 and got[1].tolist() == [-1] * tokens and got[2].tolist() == [0] * tokens
    assert got[3] is None or not bool(got[3].any())
    assert fq.fq_status() == 0


def test_a_parent_that_cannot_be_is_none(fq):
    d = [dev([0]), dev([0]), dev([4]), dev([[-1, -1]]), dev([5, 6, 7]), dev([3])]
    got = fq.fq_cache_step(*d, 4, 4, parents=dev([0, 0, 7, -3]))
    assert fq.fq_status() == -14
    assert got[2].tolist() == [0, 1, 0, 0] and got[3].tolist() == [[1], [3], [4], [8]] and got[1].tolist() == [28, 29, 30, 31]


@pytest.mark.parametrize("dt,layers,kv,dim,block,n,most,heads_first", [(torch.bfloat16, 3, 2, 64, 16, 5, 9, False), (torch.float16, 70, 1, 8, 4, 3, 40, True), (torch.float32, 1, 5, 20, 7, 40, 3, False),
                                                                       (torch.bfloat16, 2, 40, 128, 32, 2, 200, True)])
def test_move(fq, dt, layers, kv, dim, block, n, most, heads_first):
    g = torch.Generator().manual_seed(n + most)
    before, new = torch.randint(0, 30, (n,), generator=g).tolist(), torch.randint(0, most + 1, (n,), generator=g).tolist()
    new[0] = most
    lens = [a + b for a, b in zip(before, new)]
    blocks, width = sum(O.ceil_div(v, block) for v in lens) + 2, O.ceil_div(max(lens), block) + 1
    table, _ = O.make_table(lens, block, width, blocks, g)
    kept = [sorted(torch.randperm(v, generator=g)[:int(torch.randint(0, v + 1, (1,), generator=g))].tolist()) for v in new]
    kept[0] = list(range(most))[1:]              # every token moves one cell down
    if n > 2:
        kept[2] = list(range(new[2]))            # nothing moves
    shape = (blocks, kv, block, dim) if heads_first else (blocks, block, kv, dim)
    stores = [torch.randn(shape, generator=g).to(dt).cuda() for _ in range(2 * layers)]
    caches = [t.transpose(1, 2) if heads_first else t for t in stores]
    want = [t.clone() for t in caches]
    for t in want:
        old = t.clone()
        for b in range(n):
            for i, k in enumerate(kept[b]):
                src, dst = before[b] + k, before[b] + i
                t[table[b, dst // block], dst % block] = old[table[b, src // block], src % block]
    starts = [0]
    for v in new:
        starts.append(starts[-1] + v)
    wide = max(len(k) for k in kept)
    keep = fq.fq_cache_move(caches, table.cuda(), dev(starts), dev(lens), dev([k + [-5] * (wide - len(k)) for k in kept]), dev([len(k) for k in kept]))
    assert fq.fq_status() == 0 and keep.tolist() == [a + len(k) for a, k in zip(before, kept)]
    assert all(torch.equal(a, b) for a, b in zip(caches, want))


@pytest.mark.parametrize("kept,n_kept", [([2, 1], 2), ([1, 1], 2), ([0, 4], 2), ([-1, 2], 2), ([0, 1], 3), ([0, 1], -1)])
def test_a_branch_that_cannot_be_stays(fq, kept, n_kept):
    cache = torch.randn((6, 4, 2, 8), device="cuda").half()
    was = cache.clone()
    keep = fq.fq_cache_move([cache], dev([[0, 1, 2], [3, 4, 5]]), dev([0, 4, 8]), dev([7, 9]), dev([kept, [1, 3]]), dev([n_kept, 2]))
    assert fq.fq_status() == -14
    flat, old = cache.view(24, 2, 8), was.view(24, 2, 8)
    assert keep.tolist() == [3, 7]
    # sequence 0 as it was; of sequence 1 cells 6 and 8 are in cells 5 and 6
    assert torch.equal(flat[:12], old[:12])
    want = old[12:].clone()
    want[5], want[6] = old[12 + 6], old[12 + 8]
    assert torch.equal(flat[12:], want)


def test_move_refuses_blocks_outside(fq):
    cache = torch.randn((3, 4, 1, 8), device="cuda").half()
    was = cache.clone()
    keep = fq.fq_cache_move([cache], dev([[0, 3], [1, -1], [2, -1]]), dev([0, 3, 6, 7]), dev([6, 6, 2]), dev([[1, 2], [1, 2], [0, 0]]), dev([2, 2, 1]))
    assert fq.fq_status() == -14 and keep.tolist() == [3, 3, 2] and torch.equal(cache, was)
