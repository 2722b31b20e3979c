"""Sums over long rows that one CTA of 128 threads sees to alone (more rows than the SMs hold such CTAs), at values where roundings do not cancel.

A thread adds a batch of four 16-byte groups up first and its running sums once a batch: 2048 entries of fp32, 4096 of 16 bits, to a round of the
CTA's threads.  With u = 2^-24, E = sum exp(d)|d| / S and R rounds:
  a term          3 u |d|, and 4 u of its exponential
  thread          16 additions or products in a batch, R + 3 of batches (the last ones are not whole), one of the two halves of a pair
  from there on   5 steps over a warp, 2 over the warps, each after a factor off by 4 u:  15
  a rising row    a thread's sums are put on a new maximum at most once a batch, by a factor off by 4 u and a product: 5 u each
  S               u (4 + 3 E + R + 20 + 15) and 5 u R where the maximum keeps rising;  log S: as much, and 2 u of it by the logarithm
  log probability, lse, top   that, 3 u |d| and a rounding;   entropy   log S and sum exp(d) d / S, as much of E twice
The reference is a formula: all entries but one are equal, or they form a geometric series."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ROWS = 600                       # 8 CTAs on each of 148 SMs hold 1184: half of them and more, so that no row is cut
PER_ROUND = {torch.float32: 2048, torch.bfloat16: 4096, torch.float16: 4096}


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    assert c.fq_status() == 0
    c.fq_destroy()


def check(fq, z, s, e_mean, d_first, d_last, rise):
    """s, e_mean: S and E in 64 bits; d of the first and of the last entry; rise: R times what a rising maximum costs."""
    rows, vocab = z.shape
    log_s = math.log(s)
    err = 1.01 * U * (39 + 3 * e_mean + math.ceil(vocab / PER_ROUND[z.dtype]) * (1 + rise) + 2 * log_s)
    tokens = torch.zeros(rows, dtype=torch.int64, device="cuda")
    tokens[1::2] = vocab - 1
    want = torch.full((rows,), d_first - log_s, dtype=torch.float64, device="cuda")
    want[1::2] = d_last - log_s
    tol = err + 3.03 * U * max(-d_first, -d_last) + U * want.abs()
    for n_top in (0, 3):
        got, ent, ids, tops = fq.fq_token_logprobs(z, tokens, n_top)
        assert bool(((got.double() - want).abs() <= tol).all()), ("logprob", float(((got.double() - want).abs()).max()) / U, float(tol.min()) / U)
        h = log_s + e_mean
        off = float((ent.double() - h).abs().max())
        assert off <= err + 1.01 * e_mean * (2 * err + 2 * U) + U * h, ("entropy", off / U)
    # a teacher of one token: the loss is minus its log probability
    ids = tokens.int()[:, None].contiguous()
    loss, lse, _ = fq.fq_distill_topk(z, ids, torch.zeros((rows, 1), device="cuda"))
    assert bool(((loss.double() + want).abs() <= tol).all()), ("loss", float((loss.double() + want).abs().max()) / U, float(tol.min()) / U)
    assert float((lse[:, 1].double() - log_s).abs().max()) <= err
    assert torch.equal(lse[:, 0], z.float().amax(1))


@pytest.mark.parametrize("dtype", list(PER_ROUND))
@pytest.mark.parametrize("vocab", [131072, 393216])
@pytest.mark.parametrize("step", [82, 158, 203])
def test_rows_of_equal_logits_below_the_maximum(fq, dtype, vocab, step):
    """Every thread meets a logit of 0 first, then only -step / 256 (8-bit significands, so that every type holds them).  Added one by one,
    such terms lose the same part of a step each time: some 360 of 2^-24 in 393216 of them."""
    d, first = -step / 256, 4096
    z = torch.full((ROWS, vocab), d, dtype=dtype, device="cuda")
    assert float(z[0, 1]) == d
    z[:, :first] = 0.0
    s = first + (vocab - first) * math.exp(d)
    check(fq, z, s, (vocab - first) * math.exp(d) * -d / s, 0.0, d, 0)


@pytest.mark.parametrize("span", [0.02, 3.0, 100.0])
def test_rising_rows(fq, span):
    """The maximum rises all along the row: z_i = span (i / (V - 1)), formed in 64 bits and rounded to 32: what the entries' rounding does to
    the sums is in the reference, which is formed from the rounded ones."""
    vocab = 393216
    row = (torch.arange(vocab, dtype=torch.float64) * (span / (vocab - 1))).float().cuda()
    z = row.expand(ROWS, vocab).contiguous()
    d = row.double() - row.double().max()
    s = float(d.exp().sum())
    check(fq, z, s, float(-(d.exp() * d).sum()) / s, float(d[0]), float(d[-1]), 5)
