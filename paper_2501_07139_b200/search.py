"""Ensemble generation on a nested stack: builds the per-module tables with the prefill kernel and runs the
library's tree search (Sec. III-B, Algorithm 1) and pruning (Sec. III-C) on them.

The paper evaluates candidates by perplexity on a calibration set; without trained weights and datasets the
evaluation here is the relative output error of each linear layer on seeded calibration activations,
|| Y_b - Y_8 ||^2 / || Y_8 ||^2, summed over the layers of a module (and over modules for a configuration).
The attention layers of a block can be evaluated together, by what leaves the block's attention (`attention`): queries, keys and values of every precision
go through rotary positions, a paged cache and attention before the output layer, so that errors of scores count as they do in use.
The output head, whose outputs are logits, can be evaluated by what it answers instead: the divergence of its
distribution from that of the highest precision's top tokens (`head`; the search scales it to the other layers' errors),
and the perplexity of given tokens (head_answers).
The library does the heavy work: fq_gemm for the outputs, fq_sqdiff for the two fp64 sums of every comparison,
fq_cache_step, fq_rotary_cache and fq_tree_attention between them, fq_token_logprobs and fq_distill_topk for the head's, fq_code_bytes for the sizes, fq_search_chain / fq_prune_chain for
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


class Attention(NamedTuple):
    """The four layers around a block's attention, a module of their own, its heads, and how the calibration tokens are cut into sequences."""
    q: int
    k: int
    v: int
    o: int
    heads: int
    kv_heads: int
    lengths: Sequence[int]
    rotary_base: float = 10000.0
    interleaved: bool = False
    block_size: int = 64


def attention_outputs(fq: "F.FlexQ", att: Attention, shapes: Sequence, x: torch.Tensor) -> torch.Tensor:
    """What a block's attention makes of the bf16 activations `x` at the active configuration, bf16 [tokens][outputs of att.o]: every sequence is stored
    in a paged cache and sees its own tokens, each those up to itself."""
    tokens, dim, dev = x.shape[0], shapes[att.q].n_out // att.heads, x.device
    if sum(att.lengths) != tokens or shapes[att.q].n_out != att.heads * dim or shapes[att.o].k_in != att.heads * dim or any(
            shapes[i].n_out != att.kv_heads * dim for i in (att.k, att.v)):
        raise ValueError(f"attention: {att.heads} and {att.kv_heads} heads of {dim} and sequences of {sum(att.lengths)} tokens do not fit the layers and {tokens} tokens")
    q, k, v = (fq.fq_gemm(i, x, _outputs(tokens, shapes[i].n_out, dev)).view(tokens, -1, dim) for i in (att.q, att.k, att.v))
    # every sequence is new: its cache grows from nothing
    n, block = len(att.lengths), att.block_size
    width = max(1, -(-max(att.lengths) // block))
    blocks = max(1, sum(-(-t // block) for t in att.lengths))
    new = torch.tensor(list(att.lengths), dtype=torch.int32, device=dev)
    lens, free = torch.zeros_like(new), torch.arange(blocks, dtype=torch.int32, device=dev)
    table = torch.full((n, width), -1, dtype=torch.int32, device=dev)
    count = torch.full((1,), blocks, dtype=torch.int32, device=dev)
    starts, slots, positions, _ = fq.fq_cache_step(lens, lens.clone(), new, table, free, count, block, tokens)
    cache = torch.empty((2, blocks, block, att.kv_heads, dim), dtype=x.dtype, device=dev)
    turns = F.fq_rotary_table(dim, att.rotary_base, device=dev)
    q = fq.fq_rotary_cache(q, k, v, positions, slots, turns, cache[0], cache[1], interleaved=att.interleaved)
    out = fq.fq_tree_attention(q, cache[0], cache[1], table, lens, starts)
    return fq.fq_gemm(att.o, out.view(tokens, att.heads * dim), _outputs(tokens, shapes[att.o].n_out, dev))


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


def _attention_errors(fq, att, shapes, levels, x, sens_tokens, cur):
    """Sums of every level's difference from levels[0], over all tokens and over the first ones; the configuration `cur` is back in place afterwards."""
    layers, err, err_s, y_up = (att.q, att.k, att.v, att.o), [], [], None
    for b in levels:
        for i in layers:
            cur[i] = int(b)
        fq.fq_set_config(cur)
        y = attention_outputs(fq, att, shapes, x)
        if y_up is None:
            y_up = y.contiguous()
        err.append(F.fq_sqdiff(y.contiguous(), y_up))
        err_s.append(F.fq_sqdiff(y[:sens_tokens].contiguous(), y_up[:sens_tokens].contiguous()))
    for i in layers:
        cur[i] = int(levels[0])
    fq.fq_set_config(cur)
    return err, err_s


def _tables(fq, shapes, modules, levels, calib, sens_tokens, head, attention=()):
    """module_tables, and what a nat of the head's divergence counts as relative output error (1 without a head)."""
    whole = {}                           # module: its attention
    for att in attention:
        mine = [m for m, mod in enumerate(modules) if sorted(mod) == sorted((att.q, att.k, att.v, att.o))]
        if len(mine) != 1:
            raise ValueError(f"the layers {att.q}, {att.k}, {att.v}, {att.o} of an attention have to be a module of their own")
        whole[mine[0]] = att
    if head is not None and any(head.layer in mod and len(mod) > 1 for mod in modules):
        raise ValueError("the head has to be a module of its own: its error is a divergence, those of other layers are relative output errors")
    L = len(shapes)
    n_lev = len(levels)
    err = [[None] * n_lev for _ in range(L)]
    err_s = [[None] * n_lev for _ in range(L)]
    lowest = None                        # the head's error at levels[-1] as that of any other layer
    cur = [int(levels[0])] * L
    fq.fq_set_config(cur)
    whole_err = {m: _attention_errors(fq, att, shapes, levels, calib[shapes[att.q].k_in], sens_tokens, cur) for m, att in whole.items()}
    inside = {i for m in whole for i in modules[m]}
    for i, sh in enumerate(shapes):
        if i in inside:
            continue
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

    cost, sens = ([[rel(whole_err[m][which][li]) if m in whole else sum(rel(table[i][li]) for i in mod) for li in range(n_lev)]
                   for m, mod in enumerate(modules)] for which, table in enumerate((err, err_s)))
    foot = [[sum(F.fq_code_bytes(shapes[i].n_out, shapes[i].k_in, int(b)) for i in mod) for b in levels] for mod in modules]
    nats = rel(err[head.layer][-1]) if lowest is not None else 0.0
    return cost, sens, foot, rel(lowest) / nats if 0.0 < nats < math.inf else 1.0


def module_tables(fq: "F.FlexQ", shapes: Sequence, modules: Sequence[Sequence[int]], levels: Sequence[int],
                  calib: Dict[int, torch.Tensor], sens_tokens: int, head: Optional[Head] = None, attention: Sequence[Attention] = ()):
    """cost, sens, foot tables [module][level] of a stack whose layers are nested (8-bit parents).

    shapes[i] has n_out / k_in; modules[j] lists the layers of module j; levels are bit-widths from n_up down
    to n_low; calib[k_in] is a bf16 [tokens][k_in] activation matrix.  cost uses every token, sens only the
    first `sens_tokens` (the cheaper, pre-generated analysis of Sec. III-B).  `head`: that layer, a module of its own, has for its error the
    mean divergence, in nats, of its distribution from the tokens that levels[0] finds most likely.  `attention`: modules whose error is that of what leaves
    the block's attention, all four layers at a level together (without, it is the sum over the layers, each by itself).  Other rows are relative output
    errors: before rows are added up or compared, the head's wants a scale (generate_ensemble gives it one)."""
    return _tables(fq, shapes, modules, levels, calib, sens_tokens, head, attention)[:3]


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
                      prune_fraction: float = 0.0, head: Optional[Head] = None, attention: Sequence[Attention] = ()):
    """Tables, search and pruning.  With `head` the search sees the head's row of cost and sens times `head_scale`: the scale at which the divergence
    at levels[-1] counts as much as the relative output error of the head there, so that the divergence says how the head's error grows with fewer
    bits, and all rows are errors of one unit.  `cost` and `sens` are returned in the units of module_tables, `curve` is in those of the search."""
    cost, sens, foot, scale = _tables(fq, shapes, modules, levels, calib, sens_tokens, head, attention)
    weights = [scale if head is not None and head.layer in mod else 1.0 for mod in modules]
    chain, curve = F.fq_search_chain(*([[w * e for e in row] for w, row in zip(weights, table)] for table in (cost, sens)), foot, stems, branches)
    pruned, dropped, before, after = F.fq_prune_chain(chain, len(levels), foot, prune_fraction)
    return {"cost": cost, "sens": sens, "foot": foot, "chain": chain, "curve": curve, "pruned_chain": pruned,
            "dropped": dropped, "storage_before": before, "storage_after": after, "head_scale": scale}
