"""The output head evaluated by what it answers: 8-bit layers, log probabilities and distillation used together, as the ensemble generation uses
them.  The references are formed in 64 bits from the logits that the library's own product gives, so that only the
evaluation is under test; those products have tests of their own."""
from collections import namedtuple

import pytest
import torch

from fq_testlib import make_layer, to_dev, x_bf16

pytestmark = pytest.mark.gpu
Shape = namedtuple("Shape", "n_out k_in")
# log-softmax in fp32 of 1003 logits below 64: a few 2^-24 of |d| < 128 and of log S, see test_gpu_logits.py; means of some dozen rows
TOL = 2e-5


def mean_kl(ids, tops, y, t):
    lq = torch.log_softmax(y.double() / t, 1)
    lp = torch.log_softmax(tops.double(), 1)
    return (lp.exp() * (lp - lq.gather(1, ids.long()))).sum(1)


def top_of(y, t, n):
    lp = torch.log_softmax(y.double() / t, 1)
    ids = torch.sort(y.float(), dim=1, descending=True, stable=True)[1][:, :n]
    return ids, lp.gather(1, ids)


@pytest.mark.parametrize("vocab,t", [(1003, 1.0), (512, 2.0)])
def test_a_head_in_an_ensemble(vocab, t):
    import paper_2501_07139_b200 as P
    from paper_2501_07139_b200 import search as SR
    shapes = [Shape(64, 256), Shape(96, 256), Shape(vocab, 256)]
    levels, tokens, sens = [8, 5, 3], 48, 16
    fq = P.FlexQ(3)
    for i, sh in enumerate(shapes):
        c, s, z = to_dev(*make_layer(160, i, sh.n_out, sh.k_in, 8))
        fq.fq_pack_layer(i, c, s, z, 8, P.FQ_FMT_PLANES)
    x = x_bf16(160, 256, tokens, 256).cuda() * 4
    targets = torch.randint(0, vocab, (tokens,), generator=torch.Generator().manual_seed(3)).cuda()
    targets[5::9] = -1
    head = SR.Head(2, targets, n_top=20, temperature=t)
    modules = [[0, 1], [2]]
    plain = SR.module_tables(fq, shapes, modules, levels, {256: x}, sens)
    out = SR.generate_ensemble(fq, shapes, modules, levels, {256: x}, sens_tokens=sens, head=head)
    assert out["cost"][0] == plain[0][0] and out["sens"][0] == plain[1][0] and out["foot"] == plain[2]      # the others are evaluated as before
    logits = []
    for b in levels:
        fq.fq_set_config([8, 8, b])
        logits.append(fq.fq_gemm(2, x, torch.empty((tokens, 1008), dtype=torch.bfloat16, device="cuda")[:, :vocab]))
    ids, tops = top_of(logits[0], t, 20)
    assert out["cost"][1][0] == 0.0
    for li in (1, 2):
        kl = mean_kl(ids, tops, logits[li], t)
        assert abs(out["cost"][1][li] - float(kl.mean())) <= TOL and abs(out["sens"][1][li] - float(kl[:sens].mean())) <= TOL
    # the head alone; the configuration around it stays
    fq.fq_set_config([5, 3, 3])
    answers = SR.head_answers(fq, head, vocab, levels, x)
    assert [fq.fq_active_bits(i) for i in range(3)] == [5, 3, 8]
    asked = targets >= 0
    for a, y, b in zip(answers, logits, levels):
        lp = torch.log_softmax(y.double() / t, 1)
        nll = float(-lp.gather(1, targets.clamp(min=0)[:, None])[asked].mean())
        ent = float(-(lp.exp() * lp).sum(1).mean())
        assert a["bits"] == b and abs(a["nll"] - nll) <= TOL and abs(a["entropy"] - ent) <= TOL
        assert abs(a["kl"] - float(mean_kl(ids, tops, y, t).mean())) <= TOL
        assert abs(a["perplexity"] / torch.tensor(nll).double().exp().item() - 1) <= 2 * TOL
    assert fq.fq_status() == 0
    fq.fq_destroy()


def test_teacher_in_8_bits_student_in_4():
    """A step of distillation: the teacher's head in int8 gives the top tokens, the student's packed head its logits, the gradient takes their place."""
    import paper_2501_07139_b200 as P
    vocab, k, tokens, n = 1000, 512, 70, 24
    fq = P.FlexQ(1)
    w = torch.randn((vocab, k), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) * 0.02
    fq.fq_pack_layer(0, *P.fq_quantize_layer(w, 4), 4, P.FQ_FMT_PACKED)
    x = x_bf16(161, k, tokens, k).cuda() * 8
    targets = torch.arange(tokens, device="cuda") % vocab
    w8, s8 = fq.fq_quantize_rows(w)
    y8 = fq.fq_linear_i8(x, w8, s8, torch.empty((tokens, vocab), dtype=torch.float32, device="cuda"))
    lp, _, ids, tops = fq.fq_token_logprobs(y8, targets, n_top=n)
    y4 = fq.fq_gemm(0, x, torch.empty((tokens, vocab), dtype=torch.bfloat16, device="cuda"))
    kept = y4.double()
    g = torch.full((tokens,), 1.0 / tokens, device="cuda")
    loss, lse, grad = fq.fq_distill_topk(y4, ids, tops, grad_loss=g, grad=y4)
    assert grad is y4 and fq.fq_status() == 0
    # the int8 head is the exact one's up to its codes: an error of half a step per product, k of them, none of the same sign
    exact = x.double() @ w.double().T
    sx = x.double().abs().amax(1, keepdim=True) / 127
    bound = 0.5 * (sx * w.double().abs().sum(1)[None, :] + x.double().abs().sum(1, keepdim=True) * s8.double()[None, :] + 0.5 * k * sx * s8.double()[None, :])
    assert bool(((y8.double() - exact).abs() <= bound * 1.001).all())
    want_ids, want = top_of(y8, 1.0, n)
    assert torch.equal(ids, want_ids.int()) and float((tops - want).abs().max()) <= TOL
    z = kept.clone().requires_grad_()
    lq = torch.log_softmax(z, 1)
    p = torch.log_softmax(tops.double(), 1)
    ref = (p.exp() * (p - lq.gather(1, ids.long()))).sum(1)
    ref.backward(g.double())
    assert float((loss - ref.detach()).abs().max()) <= TOL
    # bf16 gradients: half a step each, and what fp32 leaves of a probability
    assert bool(((grad.double() - z.grad).abs() <= z.grad.abs() * 2.0 ** -8 + 1e-6 / tokens).all())
    fq.fq_destroy()
