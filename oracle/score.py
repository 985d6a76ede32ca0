"""float64 oracle of the scores of given tokens, one row at a time, from the definitions in the C header."""
from __future__ import annotations

import math

import numpy as np


def order(row):
    """Token ids by falling logit, equal ones by id."""
    return sorted(range(len(row)), key=lambda i: (-row[i], i))


def score(row, token, temperature=1.0, n_top=0):
    """(logprob, entropy, rank, top_ids, top_logprobs) of one row. NaN logits count as -inf, those of a magnitude of 2^126 /
    max(1, log2(e) / temperature) as infinite."""
    x = np.array(row, np.float64)
    x[np.isnan(x)] = -math.inf
    far = np.abs(x) >= 2.0 ** 126 / max(1.0, math.log2(math.e) / temperature)
    x[far] = np.sign(x[far]) * math.inf
    ids = order(x)
    some = x.max() > -math.inf
    if some:
        big = np.isinf(x) & (x > 0)
        if big.any():                                  # infinite logits share everything
            z = np.where(big, 0.0, -math.inf)
        else:
            z = (x - x.max()) / temperature
        lp = z - math.log(np.exp(z).sum())
        p = np.exp(lp)
        entropy = -float((p[p > 0] * lp[p > 0]).sum())
    else:
        lp, entropy = np.full(len(x), -math.inf), 0.0
    there = 0 <= token < len(x)
    best = [i for i in ids[:n_top] if x[i] > -math.inf]
    pad = n_top - len(best)
    return (float(lp[token]) if there else 0.0, entropy, ids.index(token) if there else -1,
            best + [-1] * pad, [float(lp[i]) for i in best] + [-math.inf] * pad)


def mean(logprobs, tokens, vocab, start):
    out = []
    for a, b in zip(start, start[1:]):
        mine = [lp for i, (lp, t) in enumerate(zip(logprobs, tokens)) if max(a, 0) <= i < b and 0 <= t < vocab]
        out.append(sum(mine) / len(mine) if mine else 0.0)
    return out
