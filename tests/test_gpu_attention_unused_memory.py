"""What lies in cells that no token uses, and infinities or NaNs among the values of a prompt, cost no time."""
import math

import pytest
import torch

from test_gpu_attention import call, make
from test_gpu_attention_odd_values import agree, defined, spoil

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    c.fq_destroy()


def filled(s, value):
    """The same sequences in caches whose other cells hold `value`."""
    out = dict(s)
    for name in ("k", "v"):
        t = s[name].clone()
        used = torch.zeros(t.shape[:2], dtype=torch.bool, device="cuda")
        for b, n in enumerate(s["lens"]):
            cells = torch.arange(n, device="cuda")
            used[s["table"][b].long()[cells // t.shape[1]], cells % t.shape[1]] = True
        t[~used] = value
        out[name] = t
    return out


def least_us(fq, s, **more):
    """The shortest of ten passes on the device."""
    lens, starts = (torch.tensor(s[n], dtype=torch.int32, device="cuda") for n in ("lens", "starts"))
    out = torch.empty_like(s["q"])
    times = []
    for _ in range(10):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        fq.fq_tree_attention(s["q"], s["k"], s["v"], s["table"], lens, starts, mask=s["mask"], out=out, **more)
        b.record()
        b.synchronize()
        times.append(1000 * a.elapsed_time(b))
    return min(times)


CASES = [([0, 0], [2000, 1990], 8, 8, 128, 64, False), ([0], [2001], 4, 4, 64, 100, False), ([500, 70], [60, 61], 16, 2, 128, 16, True), ([40], [30], 4, 1, 256, 16, False),
         ([900, 17], [3, 5], 8, 8, 128, 128, True)]


@pytest.mark.parametrize("ctx,new,heads,kv,dim,block,tree", CASES)
def test_unused_cells(fq, ctx, new, heads, kv, dim, block, tree):
    """NaN, or zeros, behind a sequence's last cell: the same bits, and no more than twice the time (a third of a launch allowed for the clock's steps)."""
    s = make(ctx, new, heads, kv, dim, block, torch.bfloat16, tree)
    zeros, nans = filled(s, 0.0), filled(s, math.nan)
    for a, b in zip(call(fq, zeros), call(fq, nans)):
        assert torch.equal(a, b)
    assert least_us(fq, nans) <= 2 * least_us(fq, zeros) + 10
    assert fq.fq_status() == 0


@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("hint", [1, 100, 2000])
def test_one_value_of_a_prompt(fq, value, hint):
    """One infinity, or NaN, among 2000 new tokens of 4 heads: twice the time is enough."""
    s = make([0], [2000], 4, 4, 128, 64, torch.bfloat16)
    clean, _ = call(fq, s, new=hint)
    for cell in (0, 700, 1990):
        hits = [(0, cell, 5, value)]
        t = spoil(s, hits)
        got, _ = call(fq, t, new=hint)
        agree(defined(t), clean, got)
        assert least_us(fq, t, new=hint) <= 2 * least_us(fq, s, new=hint) + 10
    assert fq.fq_status() == 0


@pytest.mark.parametrize("hint", [1, 100, 2000])
def test_a_prompt_of_nans(fq, hint):
    """Every value is a NaN, as a model's are that has overflowed.  A unit's cells are all noted and every row but its first sees one: some 50 thousand cycles for a unit that
    takes 10 to 30 thousand without."""
    s = make([0], [2000], 4, 4, 128, 64, torch.bfloat16)
    t = dict(s, v=torch.full_like(s["v"], math.nan))
    got, lse = call(fq, t, new=hint)
    assert bool(got[:2000].isnan().all()) and torch.equal(lse, call(fq, s, new=hint)[1])
    assert least_us(fq, t, new=hint) <= 8 * least_us(fq, s, new=hint) + 10
    assert fq.fq_status() == 0


@pytest.mark.parametrize("hint", [1, 100, 2000])
@pytest.mark.parametrize("tree", [False, True])
def test_one_column_of_a_prompt(fq, tree, hint):
    """One value of each head is infinite in every cell, of one sign and then of both: a unit notes up to 400 cells (a tree's up to 1000), which are looked at 32 at a time,
    some 2 us for 32 values of them: 100 us (250) beside the 40 that a call takes without."""
    s = make([0], [1000 if tree else 2000], 4, 4, 128, 64, torch.bfloat16, tree, words=16)
    clean, _ = call(fq, s, new=hint)
    v = s["v"].clone()
    v[..., 37] = math.inf
    both = v.clone()
    both[:, 1::2, :, 37] = -math.inf
    for t in (dict(s, v=v), dict(s, v=both)):
        got, _ = call(fq, t, new=hint)
        agree(defined(t), clean, got)
        assert least_us(fq, t, new=hint) <= 2 * least_us(fq, s, new=hint) + 500
    assert fq.fq_status() == 0


@pytest.mark.parametrize("dt,tree,value", [(torch.bfloat16, False, math.inf), (torch.float16, False, math.nan), (torch.bfloat16, True, -math.inf)])
def test_one_value_of_many(fq, dt, tree, value):
    """100 thousand new tokens, or a tree of a thousand: within the limits of the waits, and no other row changes."""
    new = 1000 if tree else 100000
    s = make([30], [new], 1, 1, 64, 64, dt, tree, words=16)
    clean, _ = call(fq, s)
    nth, d = new // 3, 11
    cell = 30 + nth
    got, _ = call(fq, spoil(s, [(0, cell, d, value)]))
    assert fq.fq_status() == 0
    rows = torch.arange(new, device="cuda")
    sees = (s["mask"][:new, nth // 64] >> (nth % 64) & 1).bool() if tree else rows >= nth
    changed = got.clone()
    changed[:new][sees, 0, d] = clean[:new][sees, 0, d]
    assert torch.equal(changed, clean)
    left = got[:new][sees, 0, d].double()
    assert bool(sees.any()) and bool((left.isnan() if math.isnan(value) else (left == value) | left.isnan()).all())
