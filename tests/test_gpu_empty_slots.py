"""Teachers padded with empty slots whose ids are out of the vocabulary."""
import math

import pytest
import torch

from test_gpu_logits import check_distill, rows_of, slots_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    assert c.fq_status() == 0
    c.fq_destroy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [40, 3001, 70001])
@pytest.mark.parametrize("wide", [False, True])
def test_an_empty_slot_may_have_any_id(fq, dtype, vocab, wide):
    """(id >= vocab, teacher -inf) is as empty as (-1, anything); with a logit of the teacher's it spoils its row."""
    rows, k = 5, 12
    z = rows_of("normal", rows, vocab, dtype, 2)
    ids, teacher, g = slots_of(rows, vocab, k, 7, wide)
    plain, padded = ids.clone(), ids.clone()
    plain[0, 7:], padded[0, 7:], teacher[0, 7:] = -1, vocab, -math.inf
    plain[1, ::2], padded[1, ::2], teacher[1, ::2] = -1, 2 ** 31 - 1, -math.inf
    if wide:
        padded[1, 2] = 2 ** 40
    plain[2], padded[2], teacher[2] = -1, vocab + 5, -math.inf                  # no slot left
    check_distill(fq, z, plain, teacher, 1.5, g)
    for upstream in (g, None):
        want, got = (fq.fq_distill_topk(z, which, teacher, 1.5, upstream) for which in (plain, padded))
        assert all(torch.equal(a, b) for a, b in zip(want, got) if a is not None)
        assert not want[0].isnan().any() and float(want[0][2]) == 0
    lse = got[1]
    assert torch.equal(*(fq.fq_distill_topk_grad(z, which, teacher, lse, g, 1.5) for which in (plain, padded)))
    teacher[3, 4], padded[3, 4] = -30.0, vocab
    loss, _, grad = fq.fq_distill_topk(z, padded, teacher, 1.5, g)
    bad = torch.tensor([False, False, False, True, False], device="cuda")
    assert torch.equal(loss.isnan(), bad) and torch.equal(grad.isnan(), bad[:, None].expand(rows, vocab))
    assert torch.equal(fq.fq_distill_topk(z, padded, teacher, 1.5)[0].isnan(), bad)
