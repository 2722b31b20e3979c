"""What lies in cells that no token uses costs no time."""
import math

import pytest
import torch

from test_gpu_attention import call, make

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
