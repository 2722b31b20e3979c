"""Attention against the definition in 64 bits, every value within what its own weights allow: a lost, doubled or misplaced cell shows."""
import math

import pytest
import torch

import fq_paged as O
from test_gpu_attention import HALF_STEP, call, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    c.fq_destroy()


def defined(s):
    """-> out, lse in 64 bits and how far each may be off.  For a row, with weights p that add up to 1:
    - scores: products of 16-bit values are exact in fp32, their sum has `dim` terms: dim + 8 roundings (tensor cores may cut off: 2^-23) of sum |q k| scale, the largest
      of the row's cells; the scale, its product and the difference from the maximum: 2^-22 of twice the largest score; the exponential 2^-21.  A weight is off by
      e of itself, and so is their sum, which has n roundings of its own;
    - weights are rounded to 16 bits: half a step of each, and with fp16 2^-25 of the largest weight where they are subnormal (the largest is 1 / sum exp(z - max));
    - the sum of n products: n + 64 roundings of sum p |v|;
    - the result is rounded: half a step."""
    q, dt = s["q"], s["q"].dtype
    tokens, heads, dim = q.shape
    block, kv = s["k"].shape[1], s["k"].shape[2]
    share, scale, h = heads // kv, dim ** -0.5, HALF_STEP[dt]
    rows = s["starts"][-1]
    out, out_off = (torch.zeros((rows, heads, dim), dtype=torch.float64, device="cuda") for _ in range(2))
    lse, lse_off = (torch.zeros((rows, heads), dtype=torch.float64, device="cuda") for _ in range(2))
    for b, length in enumerate(s["lens"]):
        r0, r1 = s["starts"][b], s["starts"][b + 1]
        n = r1 - r0
        if n == 0:
            continue
        cells = torch.arange(length, device="cuda")
        at = s["table"][b].long()[cells // block], cells % block
        nth = cells - (length - n)
        if s["mask"] is None:
            seen = nth[None] <= torch.arange(n, device="cuda")[:, None]
        else:
            seen = (nth < 0)[None] | (s["mask"][r0:r1][:, nth.clamp(min=0) // 64] >> (nth.clamp(min=0) % 64)[None] & 1).bool()
        for g in range(kv):
            k, v = s["k"][at][:, g].double(), s["v"][at][:, g].double()
            heads_of = slice(g * share, (g + 1) * share)
            x = q[r0:r1, heads_of].double()
            z = (torch.einsum("nhd,ld->nhl", x, k) * scale).masked_fill(~seen[:, None], -math.inf)
            size = (torch.einsum("nhd,ld->nhl", x.abs(), k.abs()) * scale).masked_fill(~seen[:, None], 0.0).amax(2)
            p, top = torch.softmax(z, 2), z.amax(2)
            e = (dim + 8) * 2.0 ** -23 * size + 2.0 ** -22 * 2 * size + 2.0 ** -21
            total = e + (length + 64) * 2.0 ** -24
            plus = p @ v.abs()
            o = p @ v
            off = plus * (h + e + total + (length + 64) * 2.0 ** -23)[..., None]
            if dt == torch.float16:
                off += 2.0 ** -25 * torch.exp(top - torch.logsumexp(z, 2))[..., None] * (seen.double() @ v.abs())[:, None]
            out[r0:r1, heads_of], out_off[r0:r1, heads_of] = o, 1.01 * (off + h * o.abs())
            lse[r0:r1, heads_of] = torch.logsumexp(z, 2)
            lse_off[r0:r1, heads_of] = 1.01 * (2 * total + lse[r0:r1, heads_of].abs() * 2.0 ** -22)
    return out, out_off, lse, lse_off


def within(s, want, got, lse):
    out, out_off, sums, sums_off = want
    rows = s["starts"][-1]
    assert bool(((got[:rows].double() - out).abs() <= out_off).all()), float(((got[:rows].double() - out).abs() / out_off).max())
    assert bool(((lse[:rows].double() - sums).abs() <= sums_off).all())
    assert bool((got[rows:] == 77).all()) and bool((lse[rows:] == 77).all())


LONG = [([5000], [1]), ([2500, 900, 17, 0, 70], [1, 1, 1, 1, 1]), ([3000, 129], [8, 5]), ([4100, 63], [60, 30]), ([0, 30], [1000, 700]), ([0, 0, 0], [2048, 1500, 17])]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("ctx,new", LONG)
@pytest.mark.parametrize("heads,kv,dim,block", [(2, 2, 128, 16), (8, 2, 64, 100), (4, 1, 256, 64)])
def test_long(fq, dt, ctx, new, heads, kv, dim, block):
    """Chains and prompts, cut and joined; whichever kernel `new` asks for."""
    s = make(ctx, new, heads, kv, dim, block, dt, pad=2)
    want = defined(s)
    for hint in (1, 30, 2048):
        within(s, want, *call(fq, s, new=hint))
    assert fq.fq_status() == 0


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("ctx,new", [([4100, 63], [60, 30]), ([5000, 0], [8, 8]), ([100, 700], [500, 1000])])
@pytest.mark.parametrize("heads,kv,dim,block", [(2, 2, 128, 16), (8, 2, 64, 100)])
def test_long_trees(fq, dt, ctx, new, heads, kv, dim, block):
    s = make(ctx, new, heads, kv, dim, block, dt, True, pad=2, words=16)
    want = defined(s)
    for hint in (1, 30, 2048):
        within(s, want, *call(fq, s, new=hint))
    assert fq.fq_status() == 0


@pytest.mark.parametrize("heads,kv,new,hint", [(1024, 64, 1, 1), (1024, 128, 2, 1), (1024, 1024, 16, 1), (1024, 1, 1, 100), (1024, 64, 1, 100), (1024, 8, 3, 1000), (1024, 1024, 1, 1)])
@pytest.mark.parametrize("length,block", [(1024, 16), (4003, 64), (2777, 5)])
def test_every_cell(fq, heads, kv, new, hint, length, block):
    """A row's weight lies on one cell, each row's on another: beginnings and ends of blocks and tiles, and cells all over the cache.  Its result is that cell's value, which nobody
    else has."""
    dim, dt = 128, torch.bfloat16
    if kv == 1024:
        dim = 64
    if kv * dim * length > 1 << 28:
        length //= 4
    s = make([length - new, 40], [new, new], heads, kv, dim, block, dt)
    g = torch.Generator(device="cuda").manual_seed(3)
    ends = [c for size in (block, 16, 64, 128) for c in (0, size - 1, size, 2 * size - 1, length // size * size - 1, length // size * size) if 0 <= c < length - new]
    for b, n in ((0, length), (1, 40 + new)):
        cells = torch.randint(0, n - new, (new, heads), device="cuda", generator=g)
        if b == 0:
            some = torch.tensor((ends * heads)[:heads], device="cuda")
            cells[0, ::2] = some[::2]
        block_of = s["table"][b].long()[cells // block]
        keys = s["k"][block_of, cells % block, (torch.arange(heads, device="cuda") // (heads // kv))[None]]
        # a key's own score is 3 |k|^2 / sqrt(dim), some 34 (24 of 64 values); others' are 3 times a normal number
        s["q"][s["starts"][b]:s["starts"][b + 1]] = (3 * keys.float()).to(dt)
    want = defined(s)
    within(s, want, *call(fq, s, new=hint))
    assert fq.fq_status() == 0
