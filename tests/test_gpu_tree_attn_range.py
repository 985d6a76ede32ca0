"""Attention of drafted nodes over rows in 8 bits: the bits of the probabilities, whatever the number of nodes, and scales at
both ends of float32, against the float64 oracle.

Tolerance of one output, with A = sum of p |v| over the n rows seen: as for other inputs
  A (2 d + 2^-21 + 2^-16 or 2^-24 + n 2^-24) + |o| 2^-8 or 2^-24,
(scores d, the exponential, P in two BF16 terms for BF16 or three for float32 activations, float32 sums, the output's
rounding), and for small scales what P times a row's scale loses below 2^-126, the least normal number of 32 bits: the
probabilities are carried relative to a maximum of at most the largest score, so a row adds at most |code| 2^-126 over
the sum l0 of exp(s - max s)."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2609_29499_amd import session as S
from tests.seq_case import DTYPES, flush, gen, randn, typed_cache
from tests.test_gpu_tree_attn import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("T,hq,dh", [(3, 8, 64), (17, 2, 128), (40, 2, 64), (12, 8, 128), (64, 8, 64)])
def test_probabilities_keep_sixteen_bits(kind, T, hq, dh):
    """Few rows, whose sums are often far smaller than their terms: 2^-16 of A, with any number of query rows."""
    flush(f"case bits {kind} {T} {hq} {dh}")
    lens = [0, 3, 9]
    c, kv, vv = typed_cache(lens, 1, 80, dh, kind, 60 + T)
    q = randn((3, T, hq, dh), torch.bfloat16, 61)
    got = S.tree_attention(c, 0, q.cuda())
    torch.cuda.synchronize()
    # (told that the rows are BF16, check takes P's 16 bits for its bound)
    check(got.double().cpu().numpy(), q.double().numpy(), kv[0], vv[0], lens, None, 80, "bf16", dh ** -0.5, kind="bf16")


def scored(kind, S_, H, L, powers, v_scale, seed):
    """A one-sequence cache whose row r scores powers[r] (powers of two, to the key's bits) for the query given with it:
    k has a value in its first dimension alone. v: codes of one sign, scales v_scale[r]."""
    g = gen(seed)
    dh = 64
    unit = 1.0 / 8
    k = torch.zeros((1, 1, H, S_, dh), dtype=DTYPES[kind])
    code = torch.tensor(powers, dtype=torch.float32) / unit          # small whole numbers: exact in either type
    assert torch.equal(code.to(DTYPES[kind]).float(), code)
    k[0, 0, :, :, 0] = code.to(DTYPES[kind])
    v = torch.randint(1, 128, (1, 1, H, S_, dh), generator=g).float().to(DTYPES[kind])
    ks = torch.full((1, 1, H, S_), unit)
    vs = torch.tensor(v_scale, dtype=torch.float32).expand(1, 1, H, S_).contiguous()
    c = S.SeqCache(k.cuda(), v.cuda(), torch.tensor([L], dtype=torch.int32, device="cuda"), ks.cuda(), vs.cuda())
    return c, (k.double() * ks.double()[..., None]).numpy()[0, 0], v.double().numpy()[0, 0], vs.double().numpy()[0, 0]


def check_scored(c, kv, codes, vs, L, T, hq, act, nodes, heads):
    H = kv.shape[0]
    q = torch.zeros((1, T, hq, 64), dtype=DTYPES[act])
    q[..., 0] = 1.0
    scale = math.log(2.0)
    got = S.tree_attention(c, 0, q.cuda(), scale=scale)
    torch.cuda.synchronize()
    g = got.double().cpu().numpy()
    assert np.isfinite(g).all()
    for t in nodes:
        seen = list(range(L + t + 1))
        for h in heads:
            k, vals = kv[h // (hq // H)], codes[h // (hq // H)] * vs[h // (hq // H)][:, None]
            o, A = O.attention(q[0, t, h].double().numpy(), k, vals, seen, scale)
            s = k[seen, 0] * scale
            d = 68 * 2.0 ** -24 * scale * np.abs(k[seen, 0]).max()
            tol = A * (2 * d + 2.0 ** -21 + (2.0 ** -16 if act == "bf16" else 2.0 ** -24) + len(seen) * 2.0 ** -24)
            tol = tol + np.abs(codes[h // (hq // H)][seen]).sum(0) * 2.0 ** -126 / np.exp(s - s.max()).sum()
            tol = tol + np.abs(o) * (2.0 ** -8 if act == "bf16" else 2.0 ** -24)
            assert np.all(np.abs(g[0, t, h] - o) <= tol), (t, h, float(np.max(np.abs(g[0, t, h] - o) / tol)))


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("T,hq", [(2, 2), (6, 8), (12, 8)])
def test_large_scales_under_small_probabilities(kind, act, T, hq):
    """One row far above the others holds zeros; the others, 28 powers of two below it, hold values near 10^33 (2^110: 520 of
    them, each times up to 2^8 under a running maximum, are below 2^128)."""
    flush(f"case large scales {kind} {act} {T} {hq}")
    L, S_ = 500, 520
    c, kv, codes, vs = scored(kind, S_, 1, L, [14.0] + [-14.0] * (S_ - 1), [0.0] + [2.0 ** 103] * (S_ - 1), 70)
    check_scored(c, kv, codes, vs, L, T, hq, act, sorted({0, T - 1}), [0, hq - 1])


@pytest.mark.parametrize("kind,act", [("int8", "bf16"), ("e4m3", "bf16"), ("int8", "f32")])
def test_small_scales_over_long_chunks(kind, act):
    """Values near 10^-30 in chunks of thousands of rows, most of which score 7.5 powers of two above the first ones."""
    flush(f"case small scales {kind} {act}")
    H, T, hq, L = 64, 64, 512 if act == "bf16" else 256, 8192
    S_ = L + T
    c, kv, codes, vs = scored(kind, S_, H, L, [0.0] * 64 + [7.5] * (S_ - 64), [2.0 ** -106] * S_, 71)
    check_scored(c, kv, codes, vs, L, T, hq, act, [0, 63], [0, 17, hq - 1])


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
def test_scales_over_two_hundred_powers(kind, act, order):
    """Scales from 2^-100 to 2^100 along the cache, in wide trees' kernels and in narrow ones."""
    flush(f"case scales {kind} {act} {order}")
    S_, L = 520, 500
    x = torch.linspace(-100, 100, S_).round()
    x = x[torch.randperm(S_, generator=gen(72))] if order == "mixed" else -x if order == "falling" else x
    for T, hq in ((2, 4), (12, 8)):
        c, kv, codes, vs = scored(kind, S_, 1, L, [float(r % 5) for r in range(S_)], torch.exp2(x).tolist(), 73)
        check_scored(c, kv, codes, vs, L, T, hq, act, [0, T - 1], [0, hq - 1])
