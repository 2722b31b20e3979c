"""The operators around the output head and the 8-bit layers, as cases that can be timed.

Three operators of `paper_2501_07139_b200`:

  linear    `fq_linear_i8`: activations are quantised per token to int8 and multiplied with int8 weights that carry one
            scale per output channel, Y[m][n] = sx[m] sw[n] sum_k qx[m][k] qw[n][k]
  logprobs  `fq_token_logprobs`: the log probability of one given token per row of logits, the entropy of the row and
            its most likely tokens
  distill   `fq_distill_topk` / `fq_distill_topk_grad`: the Kullback-Leibler divergence of a row's distribution from that of a
            teacher's top logits, and its gradient with respect to the logits; "pass" says which calls are made: "loss" (the
            value alone), "both" (value and gradient in one call), "apart" (the value, later the gradient from what the first
            call kept)

Where the module's `own` is false the same results come from elementary torch operations.  Linear layers have the shapes of the 7B
and 13B stacks of this repository's other cases; logits have vocabularies of generic sizes, odd ones among them.
"""
import math

import torch

own = False

FQ = None                                # the library context that a serving program keeps


def context():
    global FQ
    if FQ is None:
        import paper_2501_07139_b200 as P
        FQ = P.FlexQ(1)
    return FQ


DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # one token through an attention matrix: the latency of a decode step
        {"name": "linear-1x4096x4096", "op": "linear", "m": 1, "n": 4096, "k": 4096, "type": "fp16"},
        # eight sequences decoded together through an MLP matrix: bound by reading the weights
        {"name": "linear-8x11008x4096", "op": "linear", "m": 8, "n": 11008, "k": 4096, "type": "bf16"},
        # a short ragged prompt through the down projection
        {"name": "linear-77x4096x11008", "op": "linear", "m": 77, "n": 4096, "k": 11008, "type": "bf16"},
        # one calibration sequence through the larger stack's MLP
        {"name": "linear-2048x13824x5120", "op": "linear", "m": 2048, "n": 13824, "k": 5120, "type": "bf16"},
        # calibration-set evaluation, 4 x 2048 tokens
        {"name": "linear-8192x11008x4096", "op": "linear", "m": 8192, "n": 11008, "k": 4096, "type": "bf16"},
        # a decode step that returns the sampled token's log probability and twenty alternatives
        {"name": "logprobs-1x32000", "op": "logprobs", "rows": 1, "vocab": 32000, "type": "bf16", "top": 20, "mask": "none", "t": 1.0},
        # answers that a grammar constrains: few tokens of an odd vocabulary are left, some rows have none
        {"name": "logprobs-60x100003-grammar", "op": "logprobs", "rows": 60, "vocab": 100003, "type": "fp32", "top": 5, "mask": "grammar", "t": 0.7},
        # perplexity of two calibration sequences, the teacher's alternatives kept for distillation
        {"name": "logprobs-4094x32000", "op": "logprobs", "rows": 4094, "vocab": 32000, "type": "bf16", "top": 32, "mask": "none", "t": 1.0},
        # how far a configuration is from its parent on a short calibration text
        {"name": "distill-255x32000-loss", "op": "distill", "rows": 255, "vocab": 32000, "type": "bf16", "top": 32, "mask": "none", "t": 1.0, "pass": "loss"},
        # a training step that keeps its logits in 32 bits, the gradient asked for later
        {"name": "distill-512x50021-apart", "op": "distill", "rows": 512, "vocab": 50021, "type": "fp32", "top": 20, "mask": "none", "t": 2.0, "pass": "apart"},
        # a training step over two sequences, value and gradient at once
        {"name": "distill-4096x32000-both", "op": "distill", "rows": 4096, "vocab": 32000, "type": "bf16", "top": 32, "mask": "none", "t": 1.0, "pass": "both"},
        # the same with a large vocabulary whose last entries are padding
        {"name": "distill-1000x131072-both", "op": "distill", "rows": 1000, "vocab": 131072, "type": "bf16", "top": 64, "mask": "pad", "t": 1.5, "pass": "both"},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], evenly spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("linear", "logprobs", "distill"))
    if op == "linear":
        n, k = _spread(rng, 64, 13824), _spread(rng, 64, 13824)
        m = min(_spread(rng, 1, 8192), max(1, 8192 * 11008 * 4096 // (n * k)))
        return {"op": op, "m": m, "n": n, "k": k, "type": rng.choice(("bf16", "fp16"))}
    vocab, kind = _spread(rng, 1000, 150000), rng.choice(("bf16", "bf16", "fp16", "fp32"))
    rows = min(_spread(rng, 1, 4096), max(1, 250_000_000 // (vocab * SIZE[kind])))
    case = {"op": op, "rows": rows, "vocab": vocab, "type": kind, "t": rng.choice((1.0, 1.0, 0.7, 2.0))}
    if op == "logprobs":
        return {**case, "top": rng.choice((0, 1, 5, 20, 32, 64)), "mask": rng.choice(("none", "pad", "grammar"))}
    return {**case, "top": _spread(rng, 1, 128), "mask": rng.choice(("none", "pad")), "pass": rng.choice(("loss", "apart", "both"))}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _codes(x):
    """int8 codes and scales of the rows of x; a row's largest value becomes 127, ties go to the even code."""
    a = x.float().abs().amax(dim=1, keepdim=True)
    q = torch.round(x.double() * 127.0 / torch.where(a > 0, a, 1.0).double())
    return q, a / 127.0


def _pitched(rows, cols, dtype, device, multiple):
    """An empty matrix whose row pitch is a whole number of `multiple` elements, as 16-byte accesses need it."""
    return torch.empty((rows, -(-cols // multiple) * multiple), dtype=dtype, device=device)[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"] == "linear":
        m, n, k, dt = case["m"], case["n"], case["k"], DTYPES[case["type"]]
        x = _pitched(m, k, dt, "cuda", 8)
        x.copy_(torch.randn((m, k), device="cuda", generator=g))
        # some channels of activations are much larger than the others
        x[:, :: max(1, k // 7)] *= 12.0
        w = torch.empty((n, k), dtype=torch.float32, device="cuda").normal_(0.0, 0.02, generator=g)
        w_codes = _pitched(n, k, torch.int8, "cuda", 16)
        w_scales = torch.empty(n, dtype=torch.float32, device="cuda")
        for r in range(0, n, 4096):
            q, s = _codes(w[r:r + 4096])
            w_codes[r:r + 4096] = q.to(torch.int8)
            w_scales[r:r + 4096] = s[:, 0]
        return {"case": case, "x": x, "w_codes": w_codes, "w_scales": w_scales, "y": _pitched(m, n, dt, "cuda", 8),
                "x_codes": _pitched(m, k, torch.int8, "cuda", 16), "x_scales": torch.empty(m, dtype=torch.float32, device="cuda")}
    rows, vocab, dt, top = case["rows"], case["vocab"], DTYPES[case["type"]], case["top"]
    z = torch.randn((rows, vocab), device="cuda", generator=g).mul_(2.5)
    padding = max(1, vocab // 90) if case["mask"] == "pad" else 0        # entries that fill the vocabulary up to a round size
    tokens = torch.randint(0, vocab - padding, (rows,), device="cuda", generator=g)
    z[torch.arange(rows, device="cuda"), tokens] += 9.0 * torch.rand(rows, device="cuda", generator=g)
    if padding:
        z[:, vocab - padding:] = -math.inf
    if case["mask"] == "grammar":                    # the answer and up to some two hundred other tokens are allowed; some rows allow none
        allowed = torch.rand((rows, vocab), device="cuda", generator=g) < torch.rand((rows, 1), device="cuda", generator=g) * (200.0 / vocab)
        allowed[torch.arange(rows, device="cuda"), tokens] = True
        allowed[::13] = False
        z.masked_fill_(~allowed, -math.inf)
    if case["op"] == "logprobs":
        tokens[5::17] = -1                           # rows behind the end of a sequence
        return {"case": case, "logits": z.to(dt), "tokens": tokens}
    teacher, ids = torch.topk(z + torch.randn((rows, vocab), device="cuda", generator=g).mul_(0.5), min(top, vocab), dim=1)
    ids[3::11, ids.shape[1] // 2:] = -1              # a teacher that gave fewer
    grad_loss = torch.full((rows,), 1.0 / rows, dtype=torch.float32, device="cuda")
    grad_loss[7::19] = 0.0                           # padding
    return {"case": case, "logits": z.to(dt), "ids": ids.to(torch.int32), "teacher": teacher.contiguous(), "grad_loss": grad_loss}


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if case["op"] == "linear":
        return _own_linear(state) if own else _linear(state)
    if case["op"] == "logprobs":
        return _own_logprobs(state) if own else _logprobs(state)
    return _own_distill(state) if own else _distill(state)


def _own_linear(s):
    return context().fq_linear_i8(s["x"], s["w_codes"], s["w_scales"], s["y"], s["x_codes"], s["x_scales"])


def _own_logprobs(s):
    logprob, entropy, ids, tops = context().fq_token_logprobs(s["logits"], s["tokens"], n_top=s["case"]["top"], temperature=s["case"]["t"])
    return {"logprob": logprob, "entropy": entropy, "ids": ids, "tops": tops}


def _own_distill(s):
    fq, t, how = context(), s["case"]["t"], s["case"]["pass"]
    if how == "loss":
        return {"loss": fq.fq_distill_topk(s["logits"], s["ids"], s["teacher"], temperature=t)[0]}
    if how == "both":
        loss, _, grad = fq.fq_distill_topk(s["logits"], s["ids"], s["teacher"], temperature=t, grad_loss=s["grad_loss"])
    else:
        loss, lse, _ = fq.fq_distill_topk(s["logits"], s["ids"], s["teacher"], temperature=t)
        grad = fq.fq_distill_topk_grad(s["logits"], s["ids"], s["teacher"], lse, s["grad_loss"], temperature=t)
    return {"loss": loss, "grad": grad}


def _linear(s):
    # the quotient in 64 bits: in 32, values next to the border between two codes would fall on either side
    q, sx = _codes(s["x"])
    return ((q.float() @ s["w_codes"].float().T) * sx * s["w_scales"]).to(s["x"].dtype)


def _row_sums(z, t):
    """d = (z - max) / t, exp(d), its sum and the sum's logarithm; a row without any finite entry has d = -inf and 0, 1, 0."""
    m = z.amax(dim=1, keepdim=True)
    d = (z - torch.where(m == -math.inf, 0.0, m)) / t
    e = torch.exp(d)
    total = e.sum(dim=1, keepdim=True)
    total = torch.where(total == 0, 1.0, total)
    return d, e, total, torch.log(total)


def _logprobs(s):
    z, tokens, top = s["logits"].float(), s["tokens"], s["case"]["top"]
    d, e, total, log_total = _row_sums(z, s["case"]["t"])
    entropy = (log_total - torch.where(e > 0, e * d, 0.0).sum(dim=1, keepdim=True) / total)[:, 0]
    logprob = (d.gather(1, tokens.clamp(min=0)[:, None]) - log_total)[:, 0]
    ids = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :top]        # equal values: the lower index first
    tops = d.gather(1, ids) - log_total
    return {"logprob": torch.where(tokens < 0, 0.0, logprob), "entropy": entropy,
            "ids": torch.where(z.gather(1, ids) > -math.inf, ids, -1).to(torch.int32), "tops": tops}


def _distill(s):
    z, ids, t, how = s["logits"].float(), s["ids"].long(), s["case"]["t"], s["case"]["pass"]
    there = (ids >= 0) & (s["teacher"] > -math.inf)
    u = torch.where(there, s["teacher"], -math.inf)
    du, eu, total_u, log_u = _row_sums(u, t)
    p = eu / total_u
    d, e, total, log_total = _row_sums(z, t)
    log_q = d.gather(1, ids.clamp(min=0)) - log_total
    loss = torch.where(p > 0, p * ((du - log_u) - log_q), 0.0).sum(dim=1)
    if how == "loss":
        return {"loss": loss}
    q = e / total * there.any(dim=1, keepdim=True)
    grad = q.scatter_add(1, ids.clamp(min=0), -p) * (s["grad_loss"] / t)[:, None]
    return {"loss": loss, "grad": torch.where(s["grad_loss"][:, None] == 0, 0.0, grad).to(s["logits"].dtype)}


# ---------------------------------------------------------------------------------------------------------------- reckoning
def work(case):
    if case["op"] == "linear":
        m, n, k, e = case["m"], case["n"], case["k"], SIZE[case["type"]]
        return {"bytes": m * k * e + n * k + 4 * n + m * n * e, "flops": 2 * m * n * k}
    elements, e, rows, top = case["rows"] * case["vocab"], SIZE[case["type"]], case["rows"], case["top"]
    if case["op"] == "logprobs":
        # per entry: difference, scaling, exponential, two sums
        return {"bytes": elements * e + rows * (8 + 8 + 8 * top), "flops": 6 * elements}
    if case["pass"] == "loss":
        return {"bytes": elements * e + rows * (8 * top + 4), "flops": 4 * elements}
    reads = 2 if case["pass"] == "apart" else 1                  # two calls: the logits are read by each
    return {"bytes": (reads + 1) * elements * e + rows * (8 * top * reads + 12), "flops": 8 * elements}


def exact(case, seed):
    """From the definitions, in 64 bits: log-softmax as z / t minus the logarithm of the summed exponentials."""
    s = prepare(case, seed)
    if case["op"] == "linear":
        x = s["x"].to(torch.float64)
        largest = x.abs().max(dim=1).values
        unit = torch.where(largest > 0, largest, torch.ones_like(largest)) / 127
        steps = 127 * x / torch.where(largest > 0, largest, torch.ones_like(largest)).unsqueeze(1)
        sums = torch.matmul(steps.round(), s["w_codes"].to(torch.float64).t())
        return sums * torch.outer(unit, s["w_scales"].to(torch.float64))
    t, parts = float(case["t"]), []
    for r in range(0, case["rows"], 512):
        z = s["logits"][r:r + 512].to(torch.float64) / t
        norm = torch.logsumexp(z, dim=1, keepdim=True)
        empty = torch.isneginf(norm)
        lp = z - norm.masked_fill(empty, 0.0)                    # log probabilities; -inf throughout an empty row
        if case["op"] == "logprobs":
            tok = s["tokens"][r:r + 512]
            own_lp = lp[torch.arange(len(tok), device=tok.device), tok.clamp(min=0)].masked_fill(tok < 0, 0.0)
            weight = lp.exp()
            ent = -(weight * lp.masked_fill(torch.isneginf(lp), 0.0)).sum(1)
            best = lp.topk(case["top"], dim=1).values
            parts.append({"logprob": own_lp, "entropy": ent, "tops": best})
            continue
        ids = s["ids"][r:r + 512].long()
        u = (s["teacher"][r:r + 512].to(torch.float64) / t).masked_fill(ids < 0, -math.inf)
        lu = u - torch.logsumexp(u, dim=1, keepdim=True)
        pu = lu.exp()
        own_lq = torch.take_along_dim(lp, ids.clamp(min=0), dim=1)
        terms = torch.where(pu == 0, torch.zeros_like(pu), pu * (lu - own_lq))
        out = {"loss": terms.sum(1)}
        if case["pass"] != "loss":
            dz = lp.exp()
            dz.scatter_add_(1, ids.clamp(min=0), -pu)
            out["grad"] = dz * (s["grad_loss"][r:r + 512].to(torch.float64) / t).unsqueeze(1)
        parts.append(out)
    whole = {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
    if case["op"] == "logprobs":
        whole["ids"] = None
    return whole
