"""Paged caches for tests: the oracle of the bookkeeping in plain Python, and attention in 64 bits from the definition."""
from __future__ import annotations

import math

import torch


def ceil_div(a, b):
    return -(-a // b)


def step(lens, keep, new, table, free, count, block, tokens, parents=None, words=1):
    """fq_cache_step on lists (changed in place); returns (starts, slots, positions, bits, count)."""
    for b, row in enumerate(table):
        left, have = ceil_div(keep[b], block), ceil_div(lens[b], block)
        for j in range(left, have):
            free[count] = row[j]
            count += 1
    taken = []
    for b, row in enumerate(table):
        left, have, want = (ceil_div(v, block) for v in (keep[b], lens[b], keep[b] + new[b]))
        for j in range(left, max(have, want)):
            if j < want:
                count -= 1
                taken.append(count)
                row[j] = free[count]
            else:
                row[j] = -1
        lens[b] = keep[b] + new[b]
    starts, slots, positions, bits = [0], [], [], []
    for b, row in enumerate(table):
        first = starts[-1]
        for i in range(new[b]):
            cell = keep[b] + i
            slots.append(row[cell // block] * block + cell % block)
            branch, p = [i], parents[first + i] if parents is not None else -1
            while p >= 0:
                branch.append(p)
                p = parents[first + p]
            positions.append(keep[b] + (len(branch) - 1 if parents is not None else i))
            bits.append([sum(1 << (j - 64 * w) for j in branch if j // 64 == w) for w in range(words)])
        starts.append(first + new[b])
    behind = tokens - starts[-1]
    return starts, slots + [-1] * behind, positions + [0] * behind, bits + [[0] * words] * behind, count


def signed(bits):
    return [[v - (1 << 64) if v >> 63 else v for v in row] for row in bits]


def make_table(lens, block, width, blocks, g):
    """Table of random blocks of a cache of `blocks`; -1 behind a sequence's last."""
    order = torch.randperm(blocks, generator=g).tolist()
    return torch.tensor([[order.pop() if j < ceil_div(n, block) else -1 for j in range(width)] for n in lens], dtype=torch.int32).reshape(len(lens), width), order


def tree(n, g):
    """A parent for each of n drafted tokens."""
    return [int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(n)]


def tree_bits(parents, words):
    rows = []
    for i in range(len(parents)):
        branch, p = {i}, parents[i]
        while p >= 0:
            branch.add(p)
            p = parents[p]
        rows.append([sum(1 << (j - 64 * w) for j in branch if j // 64 == w) for w in range(words)])
    return signed(rows)


def attention(q, k, v, table, lens, starts, mask=None, scale=None):
    """-> out, lse in 64 bits, on q's device; rows behind the last new token are NaN."""
    tokens, heads, dim = q.shape
    block, kv = k.shape[1], k.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    out = torch.full((tokens, heads, dim), math.nan, dtype=torch.float64, device=q.device)
    lse = torch.full((tokens, heads), math.nan, dtype=torch.float64, device=q.device)
    for b, length in enumerate(lens):
        s0, s1 = starts[b], starts[b + 1]
        n = s1 - s0
        if n == 0:
            continue
        cells = torch.arange(length, device=q.device)
        blocks = table[b].long()[cells // block] if length else cells
        keys, values = (t[blocks, cells % block].double().repeat_interleave(heads // kv, 1) for t in (k, v))      # [length][heads][dim]
        nth = torch.arange(length, device=q.device) - (length - n)                   # which new token a cell is; negative: cached before
        if mask is None:
            seen = nth[None] <= torch.arange(n, device=q.device)[:, None]
        else:
            at = nth.clamp(0, 64 * mask.shape[1] - 1)
            seen = (mask[s0:s1][:, at // 64] >> (at % 64)[None] & 1).bool() & (nth < 64 * mask.shape[1])[None] | (nth < 0)[None]
        if length < n:
            seen = torch.zeros_like(seen)
        z = torch.einsum("nhd,lhd->hnl", q[s0:s1].double(), keys) * scale
        z = z.masked_fill(~seen, -math.inf)
        some = seen.any(1)
        p = torch.softmax(z, 2).masked_fill(~seen, 0.0)
        if bool(values.isfinite().all()):
            out[s0:s1] = torch.einsum("hnl,lhd->nhd", p, values)
        else:
            for i in range(n):                   # what a row does not see has no part in its sum, whatever it is
                out[s0 + i] = torch.einsum("hl,lhd->hd", p[:, i, seen[i]], values[seen[i]])
        lse[s0:s1] = torch.logsumexp(z, 2).T if length else -math.inf
        out[s0:s1][~some] = 0.0
        lse[s0:s1][~some] = -math.inf
    return out, lse
