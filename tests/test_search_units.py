"""The head's errors (divergences, in nats) and the other layers' (relative output errors) in one search: on tables that are made up, without a GPU."""
from collections import namedtuple
from types import SimpleNamespace

import pytest
import torch

import paper_2501_07139_b200.search as SR

Shape = namedtuple("Shape", "n_out k_in")
SHAPES = [Shape(16, 128)] * 4
LEVELS = [8, 5, 3]
# relative output errors, and divergences of the head (layer 2) in nats, at the two lower levels
REL = {0: (0.010, 0.050), 1: (0.024, 0.060), 2: (0.004, 0.030), 3: (0.016, 0.090)}
KL = (0.20, 0.50)


class Stack:
    """Outputs whose squares are the errors: y = (1, sqrt(error), 0, ...) against (1, 0, ...)."""
    n_layers = len(SHAPES)

    def __init__(self, nat):
        self.nat, self.bits = nat, [8] * len(SHAPES)

    def fq_set_config(self, bits):
        self.bits = list(bits)

    def fq_gemm(self, layer, x, y):
        y.zero_()
        y[:, 0] = 1
        level = LEVELS.index(self.bits[layer])
        if level:
            y[:, 1] = REL[layer][level - 1] ** 0.5
        self.level = level

    def fq_token_logprobs(self, y, targets, n_top, temperature):
        return None, None, torch.zeros((len(y), n_top), dtype=torch.int32), torch.zeros((len(y), n_top))

    def fq_distill_topk(self, y, ids, teacher, temperature):
        return torch.full((len(y),), KL[self.level - 1] * self.nat), None, None


@pytest.fixture
def searched(monkeypatch):
    seen = []

    def sqdiff(a, b):
        a, b = a.double(), b.double()
        return torch.stack((((a - b) ** 2).sum(), (b ** 2).sum()))

    def search(cost, sens, foot, stems, branches):
        seen.append((cost, sens))
        return real(cost, sens, foot, stems, branches)

    real = SR.F.fq_search_chain
    monkeypatch.setattr(SR.F, "fq_sqdiff", sqdiff)
    monkeypatch.setattr(SR.F, "fq_search_chain", search)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)

    def run(nat, modules=((0,), (1,), (2,), (3,)), head=True):
        x = torch.zeros((6, 128), dtype=torch.bfloat16)
        h = SR.Head(2, torch.zeros(6, dtype=torch.int64), n_top=4) if head else None
        out = SR.generate_ensemble(Stack(nat), SHAPES, modules, LEVELS, {128: x}, stems=1, branches=2, sens_tokens=2, head=h)
        return SimpleNamespace(out=out, cost=seen[-1][0], sens=seen[-1][1])

    return run


def test_the_chain_does_not_depend_on_the_unit_of_the_divergence(searched):
    runs = [searched(nat) for nat in (1.0, 1e-3, 1e3)]
    assert runs[0].out["chain"] == runs[1].out["chain"] == runs[2].out["chain"]
    for r, nat in zip(runs, (1.0, 1e-3, 1e3)):
        # what is reported of the head stays its divergence; what the search adds up is worth the head's own output error at its lowest level
        assert r.out["cost"][2] == pytest.approx([0.0, KL[0] * nat, KL[1] * nat]) and r.out["sens"][2] == pytest.approx(r.out["cost"][2])
        rel = SR.module_tables(Stack(nat), SHAPES, [[0], [1], [2], [3]], LEVELS, {128: torch.zeros((6, 128), dtype=torch.bfloat16)}, 2)[0]
        assert r.cost[2] == pytest.approx([0.0, rel[2][2] * KL[0] / KL[1], rel[2][2]]) and r.sens[2] == pytest.approx(r.cost[2])
        for m in (0, 1, 3):
            assert r.cost[m] == r.out["cost"][m] == rel[m]
        assert r.out["head_scale"] == pytest.approx(rel[2][2] / (KL[1] * nat))


def test_a_head_that_loses_nothing(searched):
    r = searched(0.0)
    assert r.cost[2] == [0.0, 0.0, 0.0] and r.out["head_scale"] == 1.0


def test_without_a_head_the_search_sees_the_tables(searched):
    r = searched(1.0, head=False)
    assert r.cost == r.out["cost"] and r.sens == r.out["sens"]


def test_a_head_is_a_module_of_its_own(searched):
    """In a module with others its error would be added to theirs."""
    with pytest.raises(ValueError, match="module of its own"):
        searched(1.0, modules=((0,), (1, 2), (3,)))
