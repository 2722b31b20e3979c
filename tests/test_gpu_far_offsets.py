"""Matrices of more than 2^31 elements or 2^32 bytes: what lies at the far end is found, and answered, as what lies in front."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_logits_far_behind():
    import paper_2501_07139_b200 as P
    rows, vocab, k = 16500, 131077, 5                          # 2.16e9 elements, 4.3e9 bytes, rows that start anywhere
    fq = P.FlexQ(1)
    z = torch.empty((rows, vocab), dtype=torch.bfloat16, device="cuda").normal_(0.0, 3.0, generator=torch.Generator(device="cuda").manual_seed(1))
    tokens = torch.arange(rows, device="cuda") * 7919 % vocab
    ids = (torch.arange(rows * k, device="cuda") * 104729 % vocab).view(rows, k)
    teacher = torch.rand((rows, k), device="cuda")
    g = torch.ones(rows, device="cuda")
    lp, ent, top, tops = fq.fq_token_logprobs(z, tokens, 3)
    loss, lse, none = fq.fq_distill_topk(z, ids, teacher)
    grad = fq.fq_distill_topk(z, ids, teacher, grad_loss=g)[2]
    later = fq.fq_distill_topk_grad(z, ids, teacher, lse, g)
    for r in (0, rows // 2, rows - 2, rows - 1):
        ref = torch.log_softmax(z[r].double(), 0)
        order = torch.sort(z[r].float(), descending=True, stable=True)[1][:3]
        assert torch.equal(top[r].long(), order)
        # a few 2^-24 of |d| < 40 and of log S < 13, twice for the difference of two of them
        assert abs(float(lp[r] - ref[tokens[r]])) < 2e-5 and abs(float(ent[r] + (ref.exp() * ref).sum())) < 1e-4
        assert float((tops[r] - ref[order]).abs().max()) < 2e-5
        p = torch.softmax(teacher[r].double(), 0)
        assert abs(float(loss[r]) - float((p * (p.log() - ref[ids[r]])).sum())) < 4e-5
        want = ref.exp()
        want.scatter_add_(0, ids[r], -p)
        for out in (grad, later):                              # half a step of bf16, and fp32's error of a probability
            assert bool(((out[r].double() - want).abs() <= want.abs() * 2.0 ** -8 + ref.exp() * 1e-5 + 1e-7).all())
    assert fq.fq_status() == 0
    fq.fq_destroy()


@pytest.mark.parametrize("m", [1, 3, 20, 300])
def test_channels_far_behind(m):
    import paper_2501_07139_b200 as P
    n, k = 1 << 20, 4112                                       # 4.3e9 weights
    fq = P.FlexQ(1)
    gen = torch.Generator(device="cuda").manual_seed(m)
    w = torch.randint(-127, 128, (n, k), dtype=torch.int8, device="cuda", generator=gen)
    sw = torch.rand(n, device="cuda", generator=gen)
    x = torch.randn((m, k), device="cuda", generator=gen).half()
    y = fq.fq_linear_i8(x, w, sw, torch.empty((m, n), dtype=torch.float32, device="cuda"))
    xc, sx = fq.fq_quantize_rows(x)
    for a in (0, n // 2, n - 128):
        ref = (xc.double() @ w[a:a + 128].double().T) * sx.double()[:, None] * sw[a:a + 128].double()
        assert bool(((y[:, a:a + 128].double() - ref).abs() <= ref.abs() * 4 * 2.0 ** -24).all())
    if m == 1:                                                 # the weights as activations: rows far behind quantised
        codes, scales = fq.fq_quantize_rows(w.view(torch.float16)[:, :1001].nan_to_num(1.0, 2.0, -2.0))
        last = w[-3:].view(torch.float16)[:, :1001].nan_to_num(1.0, 2.0, -2.0).double()
        top = last.abs().amax(1, keepdim=True)
        assert torch.equal(codes[-3:].double(), torch.round(127 * last / top)) and np.array_equal(scales[-3:].cpu().numpy(), top[:, 0].cpu().numpy().astype(np.float32) / np.float32(127))
    assert fq.fq_status() == 0
    fq.fq_destroy()
