"""The calls between the linear layers at the largest sizes, beyond 2^32 bytes, from several threads, and captured."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for path in (ROOT, os.path.join(ROOT, "tests")):
    if path not in sys.path:
        sys.path.insert(0, path)

import fq_paged as O

pytestmark = pytest.mark.gpu


def dev(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    c.fq_destroy()


@pytest.mark.parametrize("new,heads,dt", [(1, 4, torch.bfloat16), (40, 8, torch.float16), (100, 8, torch.bfloat16)])
def test_far_blocks(fq, new, heads, dt):
    """A cache whose blocks lie 2^20 values apart, over 2^31 values: the same as in a small one."""
    import paper_2501_07139_b200 as P
    g = torch.Generator(device="cuda").manual_seed(1)
    kv, dim, block, far = 2, 64, 16, 2200
    store = torch.empty(far << 20, dtype=dt, device="cuda")
    size = (far, block, kv, dim)
    big = [store.as_strided(size, (1 << 20, kv * dim, dim, 1), offset) for offset in (0, 1 << 19)]
    table_far, table_near = dev([[2199, 3, 2100, 2150, 2049, 2198, 7, 2047, 2048]]), dev([list(range(9))])
    small = [torch.zeros((9, block, kv, dim), dtype=dt, device="cuda") for _ in range(2)]
    for t in big:
        t[table_far[0].long()] = 0               # (what no token is stored in is compared too)
    lens = dev([130 if new < 100 else 140])
    starts = dev([0, new])
    before = int(lens) - new
    turns = P.fq_rotary_table(dim)
    tokens = int(lens)
    x = [torch.randn((tokens, kv, dim), device="cuda", generator=g).to(dt) for _ in range(2)]
    q = torch.randn((tokens, heads, dim), device="cuda", generator=g).to(dt)
    cell, positions = torch.arange(tokens, device="cuda"), torch.arange(tokens, device="cuda")
    outs = []
    for caches, table in ((big, table_far), (small, table_near)):
        slots = table[0].long()[cell // block] * block + cell % block
        rq = fq.fq_rotary_cache(q, x[0], x[1], positions, slots, turns, caches[0], caches[1])
        out = fq.fq_tree_attention(rq[before:], caches[0], caches[1], table, lens, starts)
        if new > 1:
            kept = [i for i in range(new) if i % 3 == 1]
            keep = fq.fq_cache_move(caches, table, starts, lens, dev([kept]), dev([len(kept)]))
            out = torch.cat((out, fq.fq_tree_attention(rq[before + kept[-1]:before + kept[-1] + 1], caches[0], caches[1], table, keep, dev([0, 1]))))
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and bool(outs[0].isfinite().all()) and fq.fq_status() == 0
    for a, b in zip(big, small):
        assert torch.equal(a[table_far[0].long()], b)


@pytest.mark.parametrize("n,tokens,most,block", [(16384, 40000, 4, 16), (3, 1 << 20, 349000, 128), (16384, 16384, 1, 1)])
def test_largest_steps(fq, n, tokens, most, block):
    g = torch.Generator().manual_seed(n)
    lens = torch.randint(0, 60, (n,), generator=g)
    keep, new = (lens * torch.rand(n, generator=g)).long(), torch.randint(0, most + 1, (n,), generator=g)
    width = (60 + most) // block + 2
    have, want = (lens + block - 1) // block, (keep + new + block - 1) // block
    blocks = int(have.sum() + want.sum()) + 1
    order = torch.randperm(blocks, generator=g).int()
    first = torch.cumsum(have, 0) - have
    col = torch.arange(width)[None]
    table = torch.where(col < have[:, None], order[(first[:, None] + col).clamp(max=blocks - 1)], -1).int()
    free = torch.cat((order[int(have.sum()):], torch.full((int(have.sum()),), -1, dtype=torch.int32)))
    d = [t.cuda() for t in (lens.int(), keep.int(), new.int(), table, free)]
    count = dev([blocks - int(have.sum())])
    got = fq.fq_cache_step(*d, count, block, tokens)
    rows, pool, ls = table.tolist(), free.tolist(), lens.tolist()
    starts, slots, positions, _, left = O.step(ls, keep.tolist(), new.tolist(), rows, pool, blocks - int(have.sum()), block, tokens)
    assert fq.fq_status() == 0 and int(count) == left and d[0].tolist() == ls and d[3].tolist() == rows
    assert torch.equal(got[0].cpu(), torch.tensor(starts, dtype=torch.int32)) and torch.equal(got[1].cpu(), torch.tensor(slots))
    assert torch.equal(got[2].cpu(), torch.tensor(positions, dtype=torch.int32)) and d[4].tolist()[:left] == pool[:left]


def test_many_caches_and_tokens(fq):
    """More caches than a launch takes, a thousand kept tokens."""
    caches = [torch.randn((70, 16, 1, 8), device="cuda").half() for _ in range(300)]
    want = [t.clone().view(1120, 1, 8) for t in caches]
    kept = list(range(1, 1025))
    for t in want:
        t[3:1027] = t[4:1028].clone()
    fq.fq_cache_move(caches, torch.arange(70, dtype=torch.int32, device="cuda")[None], dev([0, 1100]), dev([1103]), dev([kept]), dev([1024]))
    assert fq.fq_status() == 0 and all(torch.equal(a.view(1120, 1, 8), b) for a, b in zip(caches, want))


def test_scratch_that_is_too_small(fq):
    import paper_2501_07139_b200 as P
    from paper_2501_07139_b200 import flexq as F
    q, cache = torch.zeros((1, 4, 64), device="cuda").half(), torch.zeros((2, 2, 16, 4, 64), device="cuda").half()
    h, c = fq._heads(q, "q", (q.dtype,)), fq._cache(cache[0], cache[1], (q.dtype,))
    size = P.lib().fq_tree_attention_scratch(fq._h, 1, 1, 4, 4, 64, 1)
    i32, result = dev([0, 0]), torch.zeros_like(q)
    for given, code in ((size - 1, -9), (0, -9), (size, 0)):
        scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
        args = F._ATTENTION_ARGS.pack(*h, *fq._heads(result, "out", (q.dtype,)), *c, i32.data_ptr(), i32.data_ptr(), i32.data_ptr(), 2, 0, 0, scratch.data_ptr(), given,
                                      F.FQ_DT_F16, 64, 1, 1, 2, 0, 1, 1.0)
        assert P.lib().fq_tree_attention(fq._h, args, None) == code
    assert size > 0 and fq.fq_status() == 0


def calls(fq, seed, new, heads, kv):
    """A step of two sequences made from a seed, and what runs on it."""
    import paper_2501_07139_b200 as P
    g = torch.Generator().manual_seed(seed)
    gd = torch.Generator(device="cuda").manual_seed(seed)
    ctx, block, dim = [300 + seed, 40], 16, 64
    fresh = [new, max(1, new // 2)]
    lens = [a + b for a, b in zip(ctx, fresh)]
    table, rest = O.make_table(ctx, block, 40, 90, g)
    first = dict(lens=dev(ctx), table=table.cuda(), free=dev(rest + [0] * (90 - len(rest))), count=dev([len(rest)]))
    caches = torch.randn((2, 90, block, kv, dim), device="cuda", generator=gd).half()
    parents = dev([p for v in fresh for p in O.tree(v, g)])
    keep, fresh_d = dev(ctx), dev(fresh)
    qkv = [torch.randn((sum(fresh), h, dim), device="cuda", generator=gd).half() for h in (heads, kv, kv)]
    turns = P.fq_rotary_table(dim)
    kept, n_kept = dev([[0, 1], [0, 0]]), dev([min(2, new), 1])
    state = {k: v.clone() for k, v in first.items()}
    c = caches.clone()

    def reset():
        for k, v in first.items():
            state[k].copy_(v)
        c.copy_(caches)

    def run():
        reset()
        starts, slots, positions, mask = fq.fq_cache_step(state["lens"], keep, fresh_d, state["table"], state["free"], state["count"], block, sum(fresh), parents=parents,
                                                          words=-(-new // 64))
        q = fq.fq_rotary_cache(*qkv, positions, slots, turns, c[0], c[1])
        lse = torch.empty(q.shape[:2], device="cuda")
        out = fq.fq_tree_attention(q, c[0], c[1], state["table"], state["lens"], starts, mask=mask, lse=lse, new=new)
        back = fq.fq_rotary(q, qkv[1], positions, turns, inverse=True)
        left = fq.fq_cache_move([c[0], c[1]], state["table"], starts, state["lens"], kept, n_kept)
        return [starts, slots, positions, mask, q, lse, out, *back, left, c.clone(), state["table"].clone(), state["free"].clone(), state["count"].clone()]

    return run


CASES = [(1, 4, 4), (8, 8, 2), (40, 8, 2), (100, 16, 2)]


def child():
    import paper_2501_07139_b200 as P
    fq = P.FlexQ(1)
    graphs = []
    for new, heads, kv in CASES:
        run = calls(fq, new, new, heads, kv)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out, run))
    for _ in range(2):                           # all graphs one after the other, on one pool of memory each
        for graph, out, run in graphs:
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in out]
            assert all(torch.equal(a, b) for a, b in zip(got, run()))
    assert fq.fq_status() == 0
    del graphs, graph, out, run
    fq.fq_destroy()


def test_first_calls_may_be_captured():
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]


def test_several_threads(fq):
    runs = [calls(fq, 10 * i + new, new, heads, kv) for i in range(2) for new, heads, kv in CASES]
    want = [[t.clone() for t in run()] for run in runs]
    torch.cuda.synchronize()

    def work(run):
        with torch.cuda.stream(torch.cuda.Stream()):
            outs = [run() for _ in range(5)]
            torch.cuda.current_stream().synchronize()
        return outs

    with ThreadPoolExecutor(len(runs)) as pool:
        for outs, ref in zip(pool.map(work, runs), want):
            assert all(torch.equal(a, b) for out in outs for a, b in zip(out, ref))
    assert fq.fq_status() == 0


if __name__ == "__main__":
    child()
