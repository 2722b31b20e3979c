"""Ensemble generation on a nested stack: builds the per-module tables with the prefill kernel and runs the
library's tree search (Sec. III-B, Algorithm 1) and pruning (Sec. III-C) on them.

The paper evaluates candidates by perplexity on a calibration set; without trained weights and datasets the
evaluation here is the relative output error of each linear layer on seeded calibration activations,
|| Y_b - Y_8 ||^2 / || Y_8 ||^2, summed over the layers of a module (and over modules for a configuration).
The output head, whose outputs are logits, can be evaluated by what it answers instead: the divergence of its
distribution from that of the highest precision's top tokens (`head`; the search scales it to the other layers' errors),
and the perplexity of given tokens (head_answers).
The library does the heavy work: fq_gemm for the outputs, fq_sqdiff for the two fp64 sums of every comparison,
fq_token_logprobs and fq_distill_topk for the head's, fq_code_bytes for the sizes, fq_search_chain / fq_prune_chain for
the search.  This module only divides each pair of sums and adds the per-layer ratios and sizes up per module (a few
hundred host operations)."""
from __future__ import annotations

import math
from typing import Dict, List, NamedTuple, Optional, Sequence

import torch

from . import flexq as F


class Head(NamedTuple):
    """The layer whose outputs are logits, a next token for every calibration token (negative: none), and how many of the highest
    precision's tokens a lower one is held to."""
    layer: int
    targets: torch.Tensor
    n_top: int = 32
    temperature: float = 1.0


def _outputs(tokens: int, n_out: int, device) -> torch.Tensor:
    """bf16 outputs with the row pitch that fq_gemm takes."""
    return torch.empty((tokens, -(-n_out // 8) * 8), dtype=torch.bfloat16, device=device)[:, :n_out]


def head_answers(fq: "F.FlexQ", head: Head, n_out: int, levels: Sequence[int], x: torch.Tensor) -> List[dict]:
    """What the head answers to the bf16 activations `x` at every bit-width of `levels` (the other layers stay as they are, the head is left
    at levels[0]): mean negative log likelihood `nll` of the targets, its exponential `perplexity`, mean `entropy`, and `kl`, the
    mean divergence from the tokens that levels[0] finds most likely."""
    bits = [fq.fq_active_bits(i) for i in range(fq.n_layers)]
    y, out, teacher = _outputs(x.shape[0], n_out, x.device), [], None
    asked = (head.targets >= 0).sum()
    for b in list(levels) + [levels[0]]:
        bits[head.layer] = int(b)
        fq.fq_set_config(bits)
        if len(out) == len(levels):
            break
        fq.fq_gemm(head.layer, x, y)
        logprob, entropy, ids, tops = fq.fq_token_logprobs(y, head.targets, n_top=head.n_top, temperature=head.temperature)
        if teacher is None:
            # log probabilities at T: T times as much are logits (up to a constant of the row, which does not matter)
            teacher = (ids, tops * head.temperature)
        kl = fq.fq_distill_topk(y, *teacher, temperature=head.temperature)[0]
        out.append((-logprob.double().sum() / asked, entropy.double().mean(), kl.double().mean()))
    rows = torch.stack([torch.stack(o) for o in out]).tolist()
    return [{"bits": int(b), "nll": n, "perplexity": math.inf if n >= 700.0 else math.exp(n), "entropy": e, "kl": k}
            for b, (n, e, k) in zip(levels, rows)]


def _tables(fq, shapes, modules, levels, calib, sens_tokens, head):
    """module_tables, and what a nat of the head's divergence counts as relative output error (1 without a head)."""
    if head is not None and any(head.layer in mod and len(mod) > 1 for mod in modules):
        raise ValueError("the head has to be a module of its own: its error is a divergence, those of other layers are relative output errors")
    L = len(shapes)
    n_lev = len(levels)
    err = [[None] * n_lev for _ in range(L)]
    err_s = [[None] * n_lev for _ in range(L)]
    lowest = None                        # the head's error at levels[-1] as that of any other layer
    cur = [int(levels[0])] * L
    fq.fq_set_config(cur)
    for i, sh in enumerate(shapes):
        x = calib[sh.k_in]
        y_up, y = (_outputs(x.shape[0], sh.n_out, x.device) for _ in range(2))
        fq.fq_gemm(i, x, y_up)
        teacher = None
        if head is not None and i == head.layer:
            _, _, ids, tops = fq.fq_token_logprobs(y_up, head.targets, n_top=head.n_top, temperature=head.temperature)
            teacher = (ids, tops * head.temperature)
        for li, b in enumerate(levels):
            if li == 0:
                err[i][0] = err_s[i][0] = torch.zeros(2, dtype=torch.float64, device=x.device)
                continue
            cur[i] = int(b)
            fq.fq_set_config(cur)
            fq.fq_gemm(i, x, y)
            if teacher is not None:
                kl = fq.fq_distill_topk(y, *teacher, temperature=head.temperature)[0].double()
                err[i][li] = torch.stack((kl.sum(), torch.ones_like(kl).sum()))
                err_s[i][li] = torch.stack((kl[:sens_tokens].sum(), torch.ones_like(kl[:sens_tokens]).sum()))
                if li == n_lev - 1:
                    lowest = F.fq_sqdiff(y.contiguous(), y_up.contiguous())
                continue
            err[i][li] = F.fq_sqdiff(y.contiguous(), y_up.contiguous())
            err_s[i][li] = F.fq_sqdiff(y[:sens_tokens].contiguous(), y_up[:sens_tokens].contiguous())
        cur[i] = int(levels[0])
        fq.fq_set_config(cur)
    torch.cuda.synchronize()

    def rel(t):
        d2, b2 = (float(v) for v in t.cpu())
        return d2 / b2 if b2 > 0 else 0.0

    cost = [[sum(rel(err[i][li]) for i in mod) for li in range(n_lev)] for mod in modules]
    sens = [[sum(rel(err_s[i][li]) for i in mod) for li in range(n_lev)] for mod in modules]
    foot = [[sum(F.fq_code_bytes(shapes[i].n_out, shapes[i].k_in, int(b)) for i in mod) for b in levels] for mod in modules]
    nats = rel(err[head.layer][-1]) if lowest is not None else 0.0
    return cost, sens, foot, rel(lowest) / nats if 0.0 < nats < math.inf else 1.0


def module_tables(fq: "F.FlexQ", shapes: Sequence, modules: Sequence[Sequence[int]], levels: Sequence[int],
                  calib: Dict[int, torch.Tensor], sens_tokens: int, head: Optional[Head] = None):
    """cost, sens, foot tables [module][level] of a stack whose layers are nested (8-bit parents).

    shapes[i] has n_out / k_in; modules[j] lists the layers of module j; levels are bit-widths from n_up down
    to n_low; calib[k_in] is a bf16 [tokens][k_in] activation matrix.  cost uses every token, sens only the
    first `sens_tokens` (the cheaper, pre-generated analysis of Sec. III-B).  `head`: that layer, a module of its own, has for its error the
    mean divergence, in nats, of its distribution from the tokens that levels[0] finds most likely.  Other rows are relative output
    errors: before rows are added up or compared, the head's wants a scale (generate_ensemble gives it one)."""
    return _tables(fq, shapes, modules, levels, calib, sens_tokens, head)[:3]


def chain_to_bits(chain: List[List[int]], modules: Sequence[Sequence[int]], levels: Sequence[int], n_layers: int):
    """Per-layer bit vectors (what fq_set_config / fq_transition take) of a chain of module-level states."""
    out = []
    for st in chain:
        bits = [0] * n_layers
        for m, l in enumerate(st):
            for i in modules[m]:
                bits[i] = int(levels[l])
        out.append(bits)
    return out


def generate_ensemble(fq, shapes, modules, levels, calib, stems: int = 2, branches: int = 3, sens_tokens: int = 32,
                      prune_fraction: float = 0.0, head: Optional[Head] = None):
    """Tables, search and pruning.  With `head` the search sees the head's row of cost and sens times `head_scale`: the scale at which the divergence
    at levels[-1] counts as much as the relative output error of the head there, so that the divergence says how the head's error grows with fewer
    bits, and all rows are errors of one unit.  `cost` and `sens` are returned in the units of module_tables, `curve` is in those of the search."""
    cost, sens, foot, scale = _tables(fq, shapes, modules, levels, calib, sens_tokens, head)
    weights = [scale if head is not None and head.layer in mod else 1.0 for mod in modules]
    chain, curve = F.fq_search_chain(*([[w * e for e in row] for w, row in zip(weights, table)] for table in (cost, sens)), foot, stems, branches)
    pruned, dropped, before, after = F.fq_prune_chain(chain, len(levels), foot, prune_fraction)
    return {"cost": cost, "sens": sens, "foot": foot, "chain": chain, "curve": curve, "pruned_chain": pruned,
            "dropped": dropped, "storage_before": before, "storage_after": after, "head_scale": scale}
