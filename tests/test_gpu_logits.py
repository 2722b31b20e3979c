"""Log probabilities, entropies and top tokens; distillation from a teacher's top logits, value and gradient: against the definitions in 64 bits.

Tolerances, with u = 2^-24 (half a step of fp32) and d = (z - m) / T:
  exp(d)     the difference, the scaling and its constant: 3 u |d|; the exponential itself 2^-22 = 4 u
  S          those of its terms, weighted: 4 u + 3 u E where E = sum exp(d)|d| / S <= log V; additions: a thread adds at most V / 512 + 4 numbers in
             a row (two sums in each of 256 threads), the others are added in 5 + 8 + 8 steps, each after a factor of 4 u
  log S      the relative error of S, and one rounding of the result:              e = u (4 + 3 E + V / 512 + 36 + 1 + log V)
  logprob    e + 3 u |d| + u |result|
  entropy    log S and sum exp(d) d / S, whose terms are off by another u each and whose sum is too:   e + E (2 e + 2 u) + u |result|
  p of K     the same with K for V;  loss = sum p (lp - lq): sum p (e_lp + e_lq) + (the relative error of p) |lp - lq|, K additions
  gradient   g / T (q - p): relative error of q and p, products, one rounding to its type; a q, or q g / T, below 2^-126 is 0; in 16 bits
             2^(z c2 - shift) with a shift whose parts are below 64 (128 in between): four roundings of 2^-18 at most, 256 u of the
             binary logarithm of q, which is 178 u of q
All are multiplied by 1.01 for what is quadratic in u."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float16, torch.float32]
INF = math.inf
SHAPES = [(1, 1), (1, 2), (3, 7), (2, 8), (5, 100), (4, 511), (2, 1000), (4, 4097), (1, 32000), (200, 3000), (3, 32000), (2, 50021), (160, 33001),
          (2, 100003), (1, 131072), (2, 300001), (1, 393216)]


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    assert c.fq_status() == 0
    c.fq_destroy()


def rows_of(kind, rows, vocab, dtype, seed):
    """Logits of a kind, in a buffer whose rows start anywhere; what lies around them is large."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((rows, vocab), device="cuda", generator=g) * 3
    at = torch.arange(vocab, device="cuda")
    if kind == "steep":
        z *= 300
    elif kind == "ties":
        z = z.round()
    elif kind == "equal":
        z[:] = 1.25
    elif kind == "zeros":                                     # both zeros are the same value
        z = torch.where(z > 0, 0.0, -0.0)
    elif kind == "up":
        z[:] = at / vocab * 50
    elif kind == "down":
        z[:] = -at / vocab * 50
    elif kind == "few":
        z[torch.rand((rows, vocab), device="cuda", generator=g) > 3.0 / vocab] = -INF
        z[:, vocab // 2] = 1.0
    elif kind == "one":
        z[:, :] = -INF
        z[:, vocab - 1] = -7.0
    elif kind == "none":
        z[:, :] = -INF
    elif kind == "lowest":                                    # masked with the type's lowest value
        z[torch.rand((rows, vocab), device="cuda", generator=g) > 0.1] = torch.finfo(dtype).min
    elif kind == "all-lowest":
        z[:, :] = torch.finfo(dtype).min
    shift = seed % 11
    full = torch.full((rows, vocab + 13), 60000.0, dtype=dtype, device="cuda")
    full[:, shift:shift + vocab] = z.to(dtype)
    return full[:, shift:shift + vocab]


def distribution(z, t):
    """(log probabilities, probabilities, log S, E, d) in 64 bits; rows of nothing but -inf: -inf, 0, 0, 0, -inf."""
    z = z.double()
    m = z.amax(1, keepdim=True)
    d = (z - torch.where(m == -INF, 0.0, m)) / t
    s = d.exp().sum(1, keepdim=True)
    log_s = torch.where(s == 0, 0.0, s.log())
    lp = d - log_s
    p = lp.exp()
    e = (p * d.abs().nan_to_num(posinf=0.0)).sum(1)
    return lp, p, log_s[:, 0], e, d


def log_error(e, v):
    return 1.01 * U * (4 + 3 * e + v / 512 + 37 + math.log(v))


def below(got, ref, tol, what):
    # what fp32 cannot hold is an infinity there: a masked entry of -3.4e38 at T = 0.5 has the log probability -6.8e38
    ref = torch.where(ref.abs() > 2.0 ** 128 * (1 - 2.0 ** -25), ref.sign() * INF, ref)
    got = got.double()
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isnan(ref), torch.isnan(got)), what
    assert torch.equal(ref[~fin & ~torch.isnan(ref)], got[~fin & ~torch.isnan(ref)]), what
    lim = torch.broadcast_to(tol, ref.shape)
    fin &= ~(got.isinf() & (got.sign() == ref.sign()) & (ref.abs() + lim >= 2.0 ** 128 * (1 - 2.0 ** -25)))     # as near to it as the tolerance
    off, lim = (got - ref).abs()[fin], lim[fin]
    assert bool((off <= lim).all()), (what, float((off / lim.clamp(min=1e-300)).max()))


def check_logprobs(fq, z, tokens, n_top, t):
    rows, vocab = z.shape
    lp, p, log_s, e, d = distribution(z, t)
    got, ent, ids, tops = fq.fq_token_logprobs(z, tokens, n_top, t)
    err = log_error(e, vocab)
    at = tokens.clamp(min=0, max=vocab - 1).long()[:, None]
    ref, dt = lp.gather(1, at)[:, 0], d.gather(1, at)[:, 0].abs()
    ref = torch.where(tokens < 0, 0.0, ref)
    ref[tokens >= vocab] = math.nan
    below(got, ref, err + 3.03 * U * dt.nan_to_num(posinf=0.0) + U * ref.abs().nan_to_num(posinf=0.0), "logprob")
    h = log_s + e
    below(ent, h, err + 1.01 * e * (2 * err + 2 * U) + U * h, "entropy")
    if n_top:
        order = torch.sort(z.float(), dim=1, descending=True, stable=True)[1][:, :n_top]
        order = torch.nn.functional.pad(order, (0, n_top - order.shape[1]), value=0)
        there = (torch.arange(n_top, device="cuda") < vocab) & (z.float().gather(1, order) > -INF)
        assert torch.equal(ids, torch.where(there, order, -1).int())
        ref = torch.where(there, lp.gather(1, order), -INF)
        dt = d.gather(1, order).abs()
        below(tops, ref, err[:, None] + 3.03 * U * dt.nan_to_num(posinf=0.0) + U * ref.abs().nan_to_num(posinf=0.0), "top")


def tokens_of(rows, vocab, seed, dtype=torch.int64):
    return torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_logprobs_of_all_sizes(fq, dtype, rows, vocab):
    for n_top, t, seed in ((0, 1.0, 3), (5, 0.7, 4), (128, 2.0, 11)):
        check_logprobs(fq, rows_of("normal", rows, vocab, dtype, seed), tokens_of(rows, vocab, seed), n_top, t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["steep", "ties", "equal", "zeros", "up", "down", "few", "one", "none", "lowest", "all-lowest"])
def test_logprobs_of_all_kinds(fq, dtype, kind):
    for rows, vocab, n_top, t in ((1, 5, 8, 1.0), (3, 1000, 20, 0.5), (2, 33000, 1, 1.0), (2, 33000, 64, 1.0), (1, 100003, 128, 3.0)):
        check_logprobs(fq, rows_of(kind, rows, vocab, dtype, vocab % 97), tokens_of(rows, vocab, 5, torch.int32), n_top, t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9, 5000, 70001])
def test_rows_that_hold_no_numbers(fq, dtype, vocab):
    """A NaN or +inf anywhere: the row's answers are NaN, its neighbours' are not.  Tokens that ask for nothing, or for too much."""
    z = rows_of("normal", 7, vocab, dtype, 1)
    z[1, vocab - 1] = math.nan
    z[3, 0] = INF
    z[5, :] = math.nan
    tokens = torch.tensor([0, 1, -1, vocab - 1, vocab, 2, -100]).cuda()
    got, ent, ids, tops = fq.fq_token_logprobs(z, tokens, 4)
    bad = torch.tensor([False, True, False, True, False, True, False])
    assert torch.equal(ent.cpu().isnan(), bad) and torch.equal(tops.cpu().isnan(), bad[:, None].expand(7, 4))
    assert bool((ids.cpu()[bad] == -1).all()) and bool((ids.cpu()[~bad] >= 0).all())
    assert torch.equal(got.cpu().isnan(), torch.tensor([False, True, False, True, True, True, False])) and float(got[2]) == 0 and float(got[6]) == 0
    check_logprobs(fq, z[::2][:2], tokens[::2][:2].contiguous(), 4, 1.0)


# ---------------------------------------------------------------------------------------------------------------- distillation
def slots_of(rows, vocab, k, seed, wide=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.stack([torch.randperm(vocab, device="cuda", generator=g)[:k] if vocab >= k else torch.randint(0, vocab, (k,), device="cuda", generator=g)
                       for _ in range(rows)])
    teacher = torch.randn((rows, k), device="cuda", generator=g) * 2
    return ids.to(torch.int64 if wide else torch.int32), teacher, torch.rand(rows, device="cuda", generator=g) + 0.1


def check_distill(fq, z, ids, teacher, t, g, calls=("loss", "both", "apart")):
    rows, vocab = z.shape
    k = ids.shape[1]
    lp, q, log_s, e, d = distribution(z, t)
    there = (ids >= 0) & (teacher > -INF)
    some = there.any(1)
    lu, p, _, eu, du = distribution(torch.where(there, teacher, -INF), t)
    at = ids.clamp(min=0).long()
    lq, dq = lp.gather(1, at), d.gather(1, at).abs().nan_to_num(posinf=0.0)
    loss = torch.where(p > 0, p * (lu - lq), 0.0).sum(1)
    err, err_u = log_error(e, vocab)[:, None], log_error(eu, max(k, 2))[:, None]
    du = du.abs().nan_to_num(posinf=0.0)
    rel_p = err_u + (8 + 3 * du) * U
    e_term = err + err_u + 3.03 * U * (dq + du) + 3 * U * (lu.nan_to_num(neginf=0.0).abs() + lq.nan_to_num(neginf=0.0).abs())
    tol = (p * (e_term + (rel_p + (k + 4) * U) * (lu - lq).nan_to_num(posinf=0.0, neginf=0.0).abs())).sum(1) * 1.01
    grad = (q * some[:, None]).scatter_add(1, at, -p) * (g.double() / t)[:, None]
    rel_q = err + (8 + 3 * d.abs().nan_to_num(posinf=0.0) + (178 if z.dtype != torch.float32 else 0)) * U
    tol_g = (q * rel_q).scatter_add(1, at, p * (rel_p + k * U)) * (g.double() / t).abs()[:, None] * 1.02
    tol_g = tol_g + grad.abs() * (torch.finfo(z.dtype).eps / 2 + 3 * U) + {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25,
                                                                            torch.float32: 2.0 ** -126}[z.dtype]
    tol_g = tol_g + 2.0 ** -126 * (1 + (g.double() / t).abs()[:, None])
    grad[g == 0] = 0
    if "loss" in calls:
        got, lse, none = fq.fq_distill_topk(z, ids, teacher, t)
        assert none is None
        below(got, loss, tol, "loss")
        full = lse[:, 0].double() / t + lse[:, 1].double()
        want = torch.logsumexp(z.double() / t, 1)
        few = want.abs() < 1e38
        below(full[few], want[few], err[few, 0], "lse")
        assert torch.equal(lse[:, 0], z.float().amax(1))
    for how in calls:
        if how == "loss":
            continue
        around = torch.full((rows, vocab + 12), 3.0, dtype=z.dtype, device="cuda")
        out = around[:, 5:5 + vocab]
        if how == "both":
            got, lse, out2 = fq.fq_distill_topk(z, ids, teacher, t, g, out)
            below(got, loss, tol, "loss")
            assert out2 is out
        elif how == "apart":
            fq.fq_distill_topk_grad(z, ids, teacher, fq.fq_distill_topk(z, ids, teacher, t)[1], g, t, out)
        below(out, grad, tol_g, how)
        assert bool((around[:, :5] == 3).all()) and bool((around[:, 5 + vocab:] == 3).all())
    # the gradient in place of the logits, and in a matrix of its own
    full = torch.empty((rows, z.stride(0) if rows > 1 else vocab + 13), dtype=z.dtype, device="cuda")
    own = full[:, z.storage_offset() % 13:][:, :vocab]
    own.copy_(z)
    lse = fq.fq_distill_topk(own, ids, teacher, t)[1]
    fresh = fq.fq_distill_topk(z, ids, teacher, t, g)[2]
    again = own.clone()
    fq.fq_distill_topk_grad(own, ids, teacher, lse, g, t, own)
    below(own, grad, tol_g, "apart, in place")
    own.copy_(again)
    fq.fq_distill_topk(own, ids, teacher, t, g, own)
    assert torch.equal(own.nan_to_num(), fresh.nan_to_num())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_distill_of_all_sizes(fq, dtype, rows, vocab):
    for k, t, seed in ((1, 1.0, 3), (33, 0.7, 4), (128, 2.0, 11)):
        check_distill(fq, rows_of("normal", rows, vocab, dtype, seed), *slots_of(rows, vocab, k, seed, k == 33)[:2], t,
                      slots_of(rows, vocab, k, seed)[2])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["steep", "ties", "equal", "few", "one", "none", "lowest", "all-lowest"])
def test_distill_of_all_kinds(fq, dtype, kind):
    for rows, vocab, k, t in ((1, 5, 3, 1.0), (3, 1000, 20, 0.5), (2, 33000, 64, 1.0), (1, 100003, 100, 3.0)):
        ids, teacher, g = slots_of(rows, vocab, k, vocab)
        check_distill(fq, rows_of(kind, rows, vocab, dtype, vocab % 97), ids, teacher, t, g)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [40, 3001, 70001])
def test_slots(fq, dtype, vocab):
    """Empty slots, rows without any, ids that repeat, masked teachers, upstream gradients of 0 on rows that hold no numbers."""
    rows, k = 9, 12
    z = rows_of("normal", rows, vocab, dtype, 2)
    ids, teacher, g = slots_of(rows, vocab, k, 7)
    ids[0, 3:] = -1
    ids[1] = -1
    ids[2] = ids[2, 0]
    ids[3, ::2] = ids[3, 0]
    teacher[4] = -INF
    teacher[5, 1:] = -INF
    ids[6, 5] = -77
    teacher[6, 7] = -INF
    g[7] = 0.0
    teacher[8] = torch.finfo(torch.float32).min
    check_distill(fq, z, ids, teacher, 1.0, g)
    check_distill(fq, z, ids.long(), teacher, 0.5, -g)
    # rows that hold no numbers
    z[0, vocab - 1], z[1, 0], z[7, 1], z[3, 2] = math.nan, math.nan, math.nan, INF
    ids[4, 0] = vocab
    teacher[4, 0] = 0.0
    loss, lse, grad = fq.fq_distill_topk(z, ids, teacher, 1.0, g)
    later = fq.fq_distill_topk_grad(z, ids, teacher, lse, g, 1.0)
    nan = torch.zeros(rows, dtype=torch.bool, device="cuda")
    nan[[0, 3, 4, 7]] = True                                  # row 1 has no teacher
    assert torch.equal(loss.isnan(), nan) and float(loss[1]) == 0
    nan[7] = False                                            # nothing is asked of its gradient
    for out in (grad, later):
        assert bool(out[nan].isnan().all()) and not bool(out[~nan].isnan().any())
        assert bool((out[1] == 0).all()) and bool((out[7] == 0).all())
    # a slot on a masked logit: infinitely far, and the gradient asks for it with all its probability
    z = rows_of("normal", 1, vocab, dtype, 3)
    z[0, 5] = -INF
    ids = torch.tensor([[5, 6]], dtype=torch.int32).cuda()
    loss, _, grad = fq.fq_distill_topk(z, ids, torch.zeros((1, 2)).cuda(), 1.0, torch.ones(1).cuda())
    assert float(loss[0]) == INF and float(grad[0, 5]) == -0.5


@pytest.mark.parametrize("vocab", [300, 20000, 80001])
def test_gradient_against_differences(fq, vocab):
    """Central differences of the loss along directions of entries in [-1, 1]: the third derivative along one is a third central moment
    of numbers in a range of 2, at most 2^3 / (6 sqrt 3); a difference of two losses carries twice a loss's error."""
    t, h, k = 1.3, 2.0 ** -5, 24
    z = rows_of("normal", 1, vocab, torch.float32, 1)
    ids, teacher, _ = slots_of(1, vocab, k, 5)
    one = torch.ones(1, device="cuda")
    grad = fq.fq_distill_topk(z, ids, teacher, t, one)[2].double()
    for seed in range(4):
        step = torch.rand((1, vocab), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).double() * 2 - 1
        step[0, ids[0].long()] = step[0, ids[0].long()].sign()
        ends = []
        for sign in (1, -1):
            e = (z.double() + sign * h * step).float()
            ends.append((e, fq.fq_distill_topk(e, ids, teacher, t)[0].double()))
        moved = (ends[0][0].double() - ends[1][0].double()) / (2 * h)           # the step as it was after rounding
        lp = distribution(z, t)
        tol_loss = float(2 * log_error(lp[3], vocab) + 40 * U * lp[4].abs().max())
        tol = (h / t) ** 2 / 6 * 8 / (6 * math.sqrt(3)) / t + tol_loss / h + float(grad.abs().sum()) * 1e-5
        assert abs(float((ends[0][1] - ends[1][1]) / (2 * h)) - float((grad * moved).sum())) <= tol


def test_streams_and_graphs(fq):
    rows, vocab, k = 20, 40000, 16
    zs = [rows_of("normal", rows, vocab, torch.bfloat16, 11 * s + 2) for s in range(5)]       # alike in where a row starts: the same sums
    ids, teacher, g = slots_of(rows, vocab, k, 1)
    tokens = tokens_of(rows, vocab, 1)

    def calls(z):
        a = fq.fq_token_logprobs(z, tokens, 20)
        loss, lse, grad = fq.fq_distill_topk(z, ids, teacher, 1.0, g)
        return [*a, loss, lse, grad, fq.fq_distill_topk_grad(z, ids, teacher, lse, g, 1.0)]

    want = [[t.clone() for t in calls(z)] for z in zs]
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i, z in enumerate(zs):
        with torch.cuda.stream(streams[i & 1]):
            got.append(calls(z))
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(got, want))
    z = zs.pop().copy_(zs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls(z)
    for i in (1, 2, 3, 0):
        z.copy_(zs[i])
        graph.replay()
        other = calls(zs[3 - i])
        torch.cuda.synchronize()
        assert same(out, want[i]) and same(other, want[3 - i])
    del graph


def test_a_wait_that_runs_out_is_reported(fq):
    """With a limit that no copy keeps the call gives up, says so, and later ones are right."""
    rows, vocab = 300, 60000
    z = rows_of("normal", rows, vocab, torch.float32, 1)
    ids, teacher, g = slots_of(rows, vocab, 8, 1)
    fq.fq_set_wait_limit_ns(1)
    fq.fq_distill_topk(z, ids, teacher, 1.0, g)
    assert fq.fq_status() == -8
    fq.fq_set_wait_limit_ns(0)
    check_distill(fq, z, ids, teacher, 1.0, g)
    assert fq.fq_status() == 0
