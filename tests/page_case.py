"""Inputs shared by the tests of caches in pages: pools with known float64 values, shuffled tables."""
import numpy as np
import torch

from oracle import tree as O
from paper_2609_29499_amd import session as S
from tests.seq_case import DTYPES, gen


def table_of(pages, width, seed, spare=2, shared=0):
    """Tables int32 [B][width] of sequences with so many pages each, drawn from a shuffled pool (the first `shared` are the
    same for all); entries behind them are -1. Returns (table, pages of the pool)."""
    n = sum(pages) - shared * (len(pages) - 1) + spare
    order = torch.randperm(n, generator=gen(seed)).tolist()
    t = torch.full((len(pages), width), -1, dtype=torch.int32)
    at = shared
    for b, p in enumerate(pages):
        row = order[:shared] + order[at:at + p - shared]
        t[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
        at += p - shared
    return t, n


def paged(lens, counts, H, P, dh, kind, seed, layers=1, shared=0, room=0, spare=2):
    """A pool of random rows whose sequences hold lens rows and have pages for counts more (and `room` pages): the cache, and
    per sequence its rows' float64 values (k, v) [pages * P][H][dh] of every layer."""
    g = gen(seed)
    pages = [max(1, -(-(max(n, 0) + c) // P)) + room for n, c in zip(lens, counts)]
    table, n = table_of(pages, max(pages), seed, spare, shared)
    out, vals = [], []
    for _ in range(2):
        x = torch.randn((layers, n, H, P, dh), generator=g)
        x[..., ::16] *= 2.0
        x *= torch.exp2(torch.randn((layers, n, H, 1, 1), generator=g))            # pages of different sizes
        if kind == "bf16":
            t = x.to(torch.bfloat16)
            out.append((t.cuda(), None))
            vals.append(t.double())
        else:
            sc = x.abs().amax((-2, -1)) / O.QMAX[kind]
            y = (x / sc[..., None, None]).clamp(-O.QMAX[kind], O.QMAX[kind])
            t = y.round().to(torch.int8) if kind == "int8" else y.to(torch.float8_e4m3fn)
            out.append((t.cuda(), sc.cuda()))
            vals.append(t.double() * sc.double()[..., None, None])
    c = S.PageCache(out[0][0], out[1][0], table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out[0][1], out[1][1])
    rows = [[[v[la][table[b, :pages[b]].long()].permute(0, 2, 1, 3).reshape(-1, H, dh).numpy() for v in vals]
             for b in range(len(lens))] for la in range(layers)]
    return c, rows


def starts(counts, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(counts)]), dtype=torch.int32)


__all__ = ["DTYPES", "paged", "starts", "table_of"]
