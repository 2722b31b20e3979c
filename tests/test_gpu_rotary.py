"""Rotary positions against complex products in 64 bits, their gradient against autograd, and the stores to paged caches."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    c.fq_destroy()


def rates(rot, base=10000.0, factor=1.0, context=0, low=1.0, high=32.0):
    """Radians a position."""
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if context == 0:
        return [v / factor for v in f]
    kept = [min(1.0, max(0.0, (context * v / (2 * math.pi) - low) / (high - low))) for v in f]
    return [k * v + (1 - k) * v / factor for k, v in zip(kept, f)]


def turned(x, positions, rate, interleaved, magnitude=1.0, side=1.0):
    """The rotation in 64 bits."""
    x = x.double()
    rot = 2 * len(rate)
    angle = positions.double().cuda()[:, None] * torch.tensor(rate, dtype=torch.float64, device="cuda")[None] * side
    z = torch.polar(torch.full_like(angle, magnitude), angle)[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    w = torch.complex(a, b) * z
    part = torch.stack((w.real, w.imag), 3).flatten(2) if interleaved else torch.cat((w.real, w.imag), 2)
    return torch.cat((part, x[..., rot:]), 2)


def close(got, want, x, magnitude=1.0, far=0):
    """fp32 products of values, cosines (2 units of 2^-24 each, and the argument's 2^-25 half turns) and a magnitude, then one rounding.  64-bit angles
    of the reference are off by 2^-53 of themselves, themselves up to `far`."""
    size = magnitude * x.double().abs().amax(2, keepdim=True) * 1.5
    bound = want.abs() * HALF_STEP[got.dtype] + size * (8 * 2.0 ** -24 + math.pi * 2.0 ** -25 + far * 2.0 ** -52)
    return bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,kv,dim,rot", [(1, 1, 1, 2, 2), (1, 32, 32, 128, 128), (3, 7, 1, 80, 40), (5, 4, 2, 6, 6), (70, 28, 4, 96, 48), (300, 8, 8, 64, 32), (2, 3, 3, 1024, 1024), (9, 1000, 1, 16, 8),
                                                     (400, 48, 8, 128, 64)])
def test_rotary(fq, dt, interleaved, tokens, heads, kv, dim, rot):
    import paper_2501_07139_b200 as P
    g = torch.Generator(device="cuda").manual_seed(tokens + dim)
    q, k = (torch.randn((tokens, h, dim), device="cuda", generator=g).to(dt) for h in (heads, kv))
    positions = torch.randint(0, 5000, (tokens,), device="cuda", generator=g).int()
    turns = P.fq_rotary_table(rot)
    for inverse in (False, True):
        a, b = fq.fq_rotary(q, k, positions, turns, interleaved=interleaved, inverse=inverse, magnitude=1.25)
        for got, x in ((a, q), (b, k)):
            want = turned(x, positions, rates(rot), interleaved, 1.25, -1.0 if inverse else 1.0)
            assert close(got, want, x, 1.25, 5000) and torch.equal(got[..., rot:], x[..., rot:])
    assert fq.fq_rotary(q, None, positions.long(), turns, interleaved=interleaved)[1] is None
    kept = q.clone()
    a = fq.fq_rotary(kept, None, positions, turns, interleaved=interleaved, magnitude=1.25, q_out=kept)[0]      # in place
    assert a is kept and torch.equal(a, fq.fq_rotary(q, None, positions, turns, interleaved=interleaved, magnitude=1.25)[0])
    assert fq.fq_status() == 0


@pytest.mark.parametrize("scaling", [dict(), dict(factor=4.0), dict(factor=16.0, context=8192), dict(base=500000.0, factor=8.0, context=4096, low=1.0, high=4.0)])
@pytest.mark.parametrize("first", [0, 1000000, 2**31 - 40, -20, 2**40])
def test_far_positions(fq, scaling, first):
    import paper_2501_07139_b200 as P
    q = torch.randn((33, 2, 64), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    positions = first + torch.arange(33, device="cuda")
    got = fq.fq_rotary(q, None, positions, P.fq_rotary_table(64, **scaling))[0]
    # the reference's angles, in 64 bits, lose their last bits far out: integers reduce exactly here
    from fractions import Fraction
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    base, factor, context = Decimal(scaling.get("base", 10000.0)), Decimal(scaling.get("factor", 1.0)), scaling.get("context", 0)
    low, high = Decimal(scaling.get("low", 1.0)), Decimal(scaling.get("high", 32.0))
    angles = []
    for i in range(32):
        f = base ** (Decimal(-2 * i) / 64) / (2 * pi)
        kept = min(Decimal(1), max(Decimal(0), (context * f - low) / (high - low))) if context else Decimal(0)
        f = kept * f + (1 - kept) * f / factor
        angles.append([float((Fraction(f) * int(p)) % 1) * 2 * math.pi for p in positions.tolist()])
    angle = torch.tensor(angles, dtype=torch.float64, device="cuda").T[:, None]
    x, y = q.double()[..., :32], q.double()[..., 32:]
    want = torch.cat((x * angle.cos() - y * angle.sin(), x * angle.sin() + y * angle.cos()), 2)
    # (a table's fraction is off by half of 2^-64 of a turn and, before that, by 2^-62 of itself)
    bound = q.double().abs().amax(2, keepdim=True) * 1.5 * (8 * 2.0 ** -24 + math.pi * 2.0 ** -25 + abs(first) * 2.0 ** -58)
    assert bool(((got.double() - want).abs() <= bound).all())


def test_table_without_a_gpu_is_what_it_says():
    import paper_2501_07139_b200 as P
    t = P.fq_rotary_table(8, 100.0, device="cpu")
    want = [100.0 ** (-i / 4) / (2 * math.pi) for i in range(4)]
    assert all(abs(int(a) / 2.0 ** 64 - b) < 1e-15 for a, b in zip(t, want))


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(fq, interleaved):
    """The other way round is the gradient: against autograd's and against differences."""
    import paper_2501_07139_b200 as P
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((6, 3, 20), device="cuda", generator=g, dtype=torch.float64).requires_grad_()
    up = torch.randn((6, 3, 20), device="cuda", generator=g)
    positions = torch.arange(6, device="cuda").int() * 17
    (turned(x, positions, rates(12), interleaved, 1.5) * up.double()).sum().backward()
    turns = P.fq_rotary_table(12)
    got = fq.fq_rotary(up, None, positions, turns, interleaved=interleaved, inverse=True, magnitude=1.5)[0]
    assert close(got, x.grad, up, 1.5, 100)
    y = torch.randn((6, 3, 20), device="cuda", generator=g)
    step = torch.randn((6, 3, 20), device="cuda", generator=g)

    def loss(v):
        return (fq.fq_rotary(v, None, positions, turns, interleaved=interleaved, magnitude=1.5)[0].double() * up.double()).sum()

    # (linear: a difference of any size is the derivative; fp32 values of a few, 360 of them)
    assert abs(float(loss(y + step) - loss(y)) - float((got.double() * step.double()).sum())) < 360 * 30 * 2.0 ** -22


def test_strides(fq):
    """Parts of one buffer, heads before tokens, odd starts, a source that is repeated."""
    import paper_2501_07139_b200 as P
    g = torch.Generator(device="cuda").manual_seed(4)
    positions = torch.arange(11, device="cuda").int() * 9
    turns = P.fq_rotary_table(32)
    for dt in (torch.float16, torch.float32):
        wide = torch.randn((11, 1 + 5 * 32), device="cuda", generator=g).to(dt)
        views = [wide[:, 1:].view(11, 5, 32), torch.randn((5, 11, 32), device="cuda", generator=g).to(dt).transpose(0, 1),
                 torch.randn((1, 5, 36), device="cuda", generator=g).to(dt)[..., 2:34].expand(11, 5, 32), torch.randn((11, 5, 44), device="cuda", generator=g).to(dt)[..., 4:36]]
        for interleaved in (False, True):
            for v in views:
                want = fq.fq_rotary(v.contiguous(), None, positions, turns, interleaved=interleaved)[0]
                assert torch.equal(fq.fq_rotary(v, None, positions, turns, interleaved=interleaved)[0], want)
                out = torch.full((11, 5, 41), 7.0, device="cuda", dtype=dt)
                got = fq.fq_rotary(v, None, positions, turns, interleaved=interleaved, q_out=out[..., 3:35])[0]
                assert torch.equal(got, want) and bool((out[..., :3] == 7).all()) and bool((out[..., 35:] == 7).all())
    assert fq.fq_status() == 0


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,heads,kv,dim,rot,block,heads_first", [(1, 32, 32, 128, 128, 16, False), (1, 8, 2, 64, 16, 1, True), (40, 6, 2, 80, 40, 7, False), (700, 28, 4, 128, 64, 64, True), (3, 1, 1, 8, 2, 16, False)])
def test_store(fq, dt, tokens, heads, kv, dim, rot, block, heads_first):
    import paper_2501_07139_b200 as P
    g = torch.Generator(device="cuda").manual_seed(tokens + dim)
    wide = torch.randn((tokens, (heads + 2 * kv) * dim), device="cuda", generator=g).to(dt)
    q, k, v = (t.view(tokens, -1, dim) for t in wide.split([heads * dim, kv * dim, kv * dim], 1))
    positions = torch.randint(0, 9000, (tokens,), device="cuda", generator=g)
    blocks = tokens // block + 3
    slots = torch.randperm(blocks * block, device="cuda", generator=g)[:tokens]
    slots[3::5] = -1
    shape = (blocks, kv, block, dim) if heads_first else (blocks, block, kv, dim)
    caches = [torch.full(shape, 3.0 + i, device="cuda", dtype=dt) for i in range(2)]
    caches = [t.transpose(1, 2) if heads_first else t for t in caches]
    want = [t.clone().transpose(1, 2).contiguous().transpose(1, 2) if heads_first else t.clone() for t in caches]
    turns = P.fq_rotary_table(rot)
    for interleaved in (False, True):
        rq, rk = fq.fq_rotary(q, k, positions, turns, interleaved=interleaved, magnitude=0.5)
        got = fq.fq_rotary_cache(q, k, v, positions, slots, turns, *caches, interleaved=interleaved, magnitude=0.5)
        for i in range(tokens):
            s = int(slots[i])
            if s >= 0:
                want[0][s // block, s % block], want[1][s // block, s % block] = rk[i], v[i]
        assert torch.equal(got, rq) and torch.equal(caches[0], want[0]) and torch.equal(caches[1], want[1])
    same = fq.fq_rotary_cache(q, k, v, positions, slots, turns, *caches, q_out=q, magnitude=0.5)
    assert same is q and fq.fq_status() == 0


def test_a_slot_outside_is_not_followed(fq):
    import paper_2501_07139_b200 as P
    q = torch.randn((4, 2, 16), device="cuda").half()
    caches = torch.zeros((2, 3, 4, 2, 16), device="cuda").half()
    slots = torch.tensor([12, -9, 2**40, 5], device="cuda")
    fq.fq_rotary_cache(q, q, q, torch.zeros(4, dtype=torch.int32, device="cuda"), slots, P.fq_rotary_table(16), caches[0], caches[1])
    assert fq.fq_status() == -14
    flat = caches.view(2, 12, 2, 16)
    assert torch.equal(flat[0, 5], q[3]) and torch.equal(flat[1, 5], q[3])
    flat[:, 5] = 0
    assert not bool(flat.any())
