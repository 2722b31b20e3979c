"""Block numbers of a table that are no block's: each kind in a call of its own, in every kernel."""
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


@pytest.mark.parametrize("hint", [1, 60, 500])
@pytest.mark.parametrize("block", [16, 1, 5])
def test_recorded_and_read_as_zeros(fq, hint, block):
    s = make([100, 30, 60], [3, 2, 4], 4, 2, 128, block, torch.bfloat16, spare=0)
    blocks = s["k"].shape[0]
    zeroed = dict(s, k=s["k"].clone(), v=s["v"].clone())
    for t in (zeroed["k"], zeroed["v"]):
        t[int(s["table"][1, 1])] = 0
    want, lse = call(fq, zeroed, new=hint)
    assert fq.fq_status() == 0
    for number in (blocks, blocks + 1, -1, -5, 2**31 - 1, -2**31):
        bad = dict(s, table=s["table"].clone())
        bad["table"][1, 1] = number
        got, lse2 = call(fq, bad, new=hint)
        assert fq.fq_status() == -14, number
        assert torch.equal(got, want) and torch.equal(lse, lse2)
    # entries behind the sequence's last block are nobody's
    behind = dict(s, table=torch.cat((s["table"], torch.full_like(s["table"][:, :1], blocks)), 1))
    behind["table"][1][behind["table"][1] < 0] = blocks
    call(fq, behind, new=hint)
    assert fq.fq_status() == 0
