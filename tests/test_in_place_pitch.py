"""A gradient in place of the logits has their pitch: refused otherwise, before the context or a pointer is looked into."""
import pytest

import paper_2501_07139_b200 as P
from test_head_refusals import ARG, BUF, DISTILL, GRAD, PAGE


@pytest.mark.parametrize("name,args", [("fq_distill_topk", DISTILL), ("fq_distill_topk_grad", GRAD)])
@pytest.mark.parametrize("ld,ldg", [(100, 104), (104, 100)])
def test_refused(name, args, ld, ldg):
    args = {**args, "ld": ld, "ldg": ldg}
    assert args["z"] == args["grad"] == BUF
    assert getattr(P.lib(), name)(*args.values()) == ARG
    assert PAGE.raw == bytes(1 << 16)
