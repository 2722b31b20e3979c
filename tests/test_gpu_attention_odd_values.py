"""Infinities and NaNs among cached values: every row sees them, wherever the new tokens begin in a block or a tile."""
import math

import pytest
import torch

import fq_paged as O
from test_gpu_attention import call, make

pytestmark = pytest.mark.gpu
VALUES = (math.nan, math.inf, -math.inf)


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    c.fq_destroy()


def spoil(s, hits):
    """The caches with values replaced: hits = (sequence, cell, column, value), in the last key head."""
    v = s["v"].clone()
    block = v.shape[1]
    for b, cell, d, x in hits:
        v[int(s["table"][b, cell // block]), cell % block, -1, d] = x
    return dict(s, v=v)


def defined(s):
    return O.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["starts"], s["mask"])[0][:s["starts"][-1]]


def agree(want, clean, got):
    """Where the definition is finite nothing changes, elsewhere the result is infinite, with the definition's sign, or NaN."""
    got, clean, fine = got[:len(want)], clean[:len(want)], want.isfinite()
    assert not bool(fine.all())
    assert torch.equal(got[fine], clean[fine])
    left = got[~fine].double()
    assert not bool(left.isfinite().any())
    assert bool((left.isnan() | (left == want[~fine])).all())


# up to 16 rows a key head: 1, 2, 8, 16; more: 20, 64, 320
ROWS = [(4, 4, 1), (8, 4, 1), (2, 2, 8), (16, 2, 2), (16, 4, 5), (64, 2, 2), (64, 2, 10)]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv,new", ROWS)
def test_cached_values(fq, dt, tree, dim, heads, kv, new):
    """One value of a sequence, 0 .. 17 cells before its new tokens, which begin anywhere in a tile of 16."""
    ctx = [d + 1 + (0, 16, 5, 130, 251)[d % 5] for d in range(18)] + [1000, 3]
    s = make(ctx, [new] * 20, heads, kv, dim, 16, dt, tree, words=1)
    clean, lse = call(fq, s)
    for x in VALUES:
        hits = [(b, ctx[b] - 1 - b, 3 + b, x) for b in range(18)]
        t = spoil(s, hits)
        got, lse2 = call(fq, t)
        agree(defined(t), clean, got)
        assert torch.equal(lse, lse2)
    assert fq.fq_status() == 0


@pytest.mark.parametrize("heads,kv,new", ROWS)
@pytest.mark.parametrize("tree", [False, True])
def test_cached_and_new_values(fq, heads, kv, new, tree):
    """Both in one tile, of both signs, whichever kernel the number of new tokens asks for; single sequences, whose work is cut, and many, whose work is whole."""
    for n in (1, 3, 600):
        ctx = [(37 * b) % 83 + 2 for b in range(n)]
        s = make(ctx, [new] * n, heads, kv, 64, 16, torch.bfloat16, tree, words=1)
        hits = []
        for b in range(0, n, 2):
            hits += [(b, ctx[b] - 1, 5, math.inf), (b, ctx[b] - 2, 6, math.nan), (b, ctx[b] + b % new, 5, -math.inf), (b, ctx[b] + new - 1, 9, math.inf)]
        t = spoil(s, hits)
        want = defined(t)
        for hint in (None, 1, 30, 500):
            clean, _ = call(fq, s, new=hint)
            got, _ = call(fq, t, new=hint)
            agree(want, clean, got)
    assert fq.fq_status() == 0


@pytest.mark.parametrize("length", [4003, 4007, 4015, 4016])
@pytest.mark.parametrize("hint", [1, 100])
def test_long_cache(fq, length, hint):
    """One token; its cache is every worker's."""
    s = make([length - 1], [1], 4, 4, 128, 16, torch.float16)
    clean, _ = call(fq, s, new=hint)
    for back in (1, 2, 3, 7, 16, 1000, length - 1):
        hits = [(0, length - 1 - back, 7, math.inf)]
        t = spoil(s, hits)
        got, _ = call(fq, t, new=hint)
        agree(defined(t), clean, got)
    assert fq.fq_status() == 0


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("hint", [1, 4, 30, 500])
@pytest.mark.parametrize("tree", [False, True])
def test_new_values_by_every_kernel(fq, dt, hint, tree):
    """Values of new tokens touch the rows that see them, and no others."""
    s = make([50, 0, 131, 16], [9, 40, 70, 1], 4, 2, 128, 16, dt, tree, words=2)
    clean, _ = call(fq, s, new=hint)
    for x in VALUES:
        hits = [(0, 54, 3, x), (1, 33, 3, x), (1, 39, 120, -x), (2, 131, 64, x), (2, 200, 3, x), (2, 181, 3, -x), (3, 16, 0, x)]
        t = spoil(s, hits)
        got, _ = call(fq, t, new=hint)
        agree(defined(t), clean, got)
    assert fq.fq_status() == 0
