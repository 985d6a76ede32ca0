"""Inputs shared by the drafted-token GPU tests: typed caches with known float64 values, random trees."""
import numpy as np
import torch

from oracle import tree as O
from paper_2609_29499_amd import session as S

DTYPES = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn, "f32": torch.float32}


def flush(msg):
    print(msg, flush=True)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def random_parents(B, T, seed, width=6, absent=True):
    """Trees int32 [B][T]; every third sequence misses its last nodes, and one node in the middle."""
    rng = np.random.default_rng(seed)
    p = np.full((B, T), -1, np.int32)
    for b in range(B):
        for t in range(1, T):
            p[b, t] = rng.integers(max(0, t - width), t)
        if absent and b % 3 == 2:
            p[b, max(1, T - T // 3):] = -2
            if T > 6:
                p[b, 4] = 99
    return torch.from_numpy(p)


def typed_cache(lens, H, S_, dh, kind, seed, layers=1):
    """A cache of random rows on the GPU and its values in float64 numpy [L][B][H][S][dh]."""
    g = gen(seed)
    B = len(lens)
    out, vals = [], []
    for _ in range(2):
        x = torch.randn((layers, B, H, S_, dh), generator=g)
        x[..., ::16] *= 2.0
        if kind == "bf16":
            t = x.to(torch.bfloat16)
            out.append((t.cuda(), None))
            vals.append(t.double().numpy())
        else:
            sc = x.abs().amax(-1) / O.QMAX[kind]
            y = (x / sc[..., None]).clamp(-O.QMAX[kind], O.QMAX[kind])
            t = y.round().to(torch.int8) if kind == "int8" else y.to(torch.float8_e4m3fn)
            out.append((t.cuda(), sc.cuda()))
            vals.append(t.double().numpy() * sc.double().numpy()[..., None])
    c = S.SeqCache(out[0][0], out[1][0], torch.tensor(lens, dtype=torch.int32, device="cuda"), out[0][1], out[1][1])
    return c, vals[0], vals[1]


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=gen(seed)).to(dtype)
