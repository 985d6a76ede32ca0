"""Causal attention of packed tokens over pages against the float64 oracle.

Tolerance of one output: with A = sum of p |v| over the rows seen, n their number,
  scores: a float32 dot product of dh exact products, |error| <= (dh + 4) 2^-24 scale sum |q_i k_i| = d, which
  moves p by a factor within exp(2 d);
  exp2 and the rescaling by powers: 2^-21; P in two BF16 terms 2^-16, in three 2^-24; more than 32 BF16 query rows of a sequence and cache head: one FP16 term, half a step 2^-11, and half a step
  of FP16's least numbers, 2^-25, of P (lifted by 2^10; V times it is in units of the largest |v| or less) and of V (the largest at
  2^11 or more): n (2^-35 + 2^-36) max |v|, less than n 2^-34 max |v| together;
  float32 sums n 2^-24;
  the output's rounding 2^-8 of the value in BF16, 2^-24 in float32.
|error| <= A (2 d + 2^-21 + 2^-11, 2^-16 or 2^-24 + n 2^-24) + (n 2^-34 max |v|) + |o| 2^-8 or 2^-24."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2609_29499_amd import session as S
from tests.page_case import paged, starts
from tests.seq_case import DTYPES, flush, gen, randn

pytestmark = pytest.mark.gpu


def check(got, q, rows, lens, counts, P, act, scale, first=0, cap=None, gone=lambda b, r: False, some=None):
    """got [N][Hq][dh] float64 against the oracle; gone(b, r): row r of sequence b has no page. some: tokens of a sequence that are looked at."""
    N, hq, dh = q.shape
    worst = 0.0
    t0 = first
    for b, (L, c) in enumerate(zip(lens, counts)):
        H = rows[b][0].shape[1]
        G = hq // H
        half = act == "bf16" and c * G > 32
        for i in range(c) if some is None else sorted({x for x in some(c) if 0 <= x < c}):
            t = t0 + i
            seen = [] if L < 0 or (cap is not None and (L > cap or L + i >= cap)) else [r for r in range(L + i + 1) if not gone(b, r)]
            if not seen:
                assert not got[t].any(), (b, i)
                continue
            for h in range(hq):
                k, v = rows[b][0][:, h // G], rows[b][1][:, h // G]
                o, A = O.attention(q[t, h], k, v, seen, scale)
                d = (dh + 4) * 2.0 ** -24 * scale * np.max(np.abs(k[seen]) @ np.abs(q[t, h]))
                tol = A * (2 * d + 2.0 ** -21 + (2.0 ** -11 if half else 2.0 ** -16 if act == "bf16" else 2.0 ** -24) + len(seen) * 2.0 ** -24)
                tol = tol + half * len(seen) * 2.0 ** -34 * np.max(np.abs(v[seen]))
                tol = tol + np.abs(o) * (2.0 ** -8 if act == "bf16" else 2.0 ** -24)
                err = np.abs(got[t, h] - o)
                worst = max(worst, float(np.max(np.divide(err, tol, out=np.zeros_like(err), where=tol > 0))))
                assert np.all(err <= tol), (b, i, h, float(np.max(err / tol)))
        t0 += c
    flush(f"   worst share of the tolerance {worst:.3f}")


CASES = [
    # lens, counts (None: one each, without start), P, hq, hkv, dh, cache, act
    ([0], None, 16, 4, 4, 64, "bf16", "bf16"),
    ([1], None, 128, 8, 1, 128, "int8", "bf16"),
    ([0, 5, 31], [3, 1, 2], 16, 6, 3, 64, "int8", "bf16"),
    ([32, 31, 33, 0], [5, 0, 7, 1], 32, 8, 2, 128, "e4m3", "bf16"),
    ([127, 128, 129], [16, 2, 1], 64, 4, 1, 128, "bf16", "bf16"),
    ([300, 0, 17], [64, 70, 3], 16, 8, 1, 128, "int8", "bf16"),
    ([77, 500], [33, 1], 32, 9, 3, 64, "bf16", "f32"),
    ([600], [7], 128, 28, 4, 128, "e4m3", "f32"),
    ([2000, 3, 900, 0, 1500], None, 64, 16, 2, 64, "e4m3", "bf16"),
    ([4100], None, 16, 4, 1, 64, "int8", "f32"),
    ([0], [333], 64, 8, 2, 64, "bf16", "bf16"),
    ([0, 100], [130, 200], 16, 16, 2, 128, "e4m3", "bf16"),
    ([65], [257], 32, 3, 1, 64, "int8", "f32"),
    ([1000, 10, 0], [150, 1, 1], 64, 5, 1, 128, "int8", "bf16"),
    ([50 * i for i in range(40)], None, 16, 7, 1, 64, "int8", "bf16"),
]


def edges(c):
    """Tokens of a long list that are looked at."""
    return range(c) if c < 12 else [0, 1, 7, 8, 15, 16, 31, 32, 33, 63, 64, c // 2, c - 2, c - 1]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_page_attention(case):
    lens, counts, P, hq, H, dh, kind, act = CASES[case]
    flush(f"case attention {CASES[case]}")
    n = [1] * len(lens) if counts is None else counts
    c, rows = paged(lens, n, H, P, dh, kind, case)
    q = randn((sum(n), hq, dh), DTYPES[act], 100 + case)
    got = S.page_attention(c, 0, q.cuda(), None if counts is None else starts(n).cuda())
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, n, P, act, dh ** -0.5, some=edges)


@pytest.mark.parametrize("kind,counts,hq,dh,P", [("bf16", [3, 1, 2, 1], 4, 128, 16), ("int8", [1, 1, 1, 1], 4, 128, 64), ("e4m3", [9, 2, 5, 1], 8, 64, 128),
                                                 ("int8", [40, 1, 20, 12], 8, 128, 32), ("bf16", [100, 3, 1, 64], 8, 64, 64),
                                                 ("e4m3", [64, 0, 300, 1], 16, 128, 16)])
def test_long_contexts_in_many_chunks(kind, counts, hq, dh, P):
    """Ragged sequences over several chunks, hints that are too small or too large, strided q and out, tokens of no
    sequence, a shared prefix."""
    lens = [20000, 700, 300, 9001]
    flush(f"case long {kind} {counts} {hq} {dh} {P}")
    H, front, behind = 2, 4, 3
    c, rows = paged(lens, counts, H, P, dh, kind, 7, shared=300 // P)
    N = front + sum(counts) + behind
    wide = torch.full((N, 3, hq, dh), math.nan, dtype=torch.bfloat16, device="cuda")
    q = randn((N, hq, dh), torch.bfloat16, 8)
    wide[front:N - behind, 1] = q[front:N - behind].cuda()
    out = torch.full((N, hq + 1, dh), 5.0, dtype=torch.bfloat16, device="cuda")
    at = starts(counts, front).cuda()
    for max_len, max_new in ((20000, max(counts)), (4000, 1), (100, N), (c.max_seq, 2)):
        out.fill_(5.0)
        S.page_attention(c, 0, wide[:, 1], at, max_len=max_len, max_new=max_new, out=out[:, :hq])
        torch.cuda.synchronize()
        check(out[:, :hq].double().cpu().numpy(), q.double().numpy(), rows[0], lens, counts, P, "bf16", dh ** -0.5, first=front,
              some=lambda c: [0, c // 2, c - 1])
        assert torch.all(out[:, hq] == 5.0) and torch.all(out[:front] == 5.0) and torch.all(out[N - behind:] == 5.0)
        again = torch.full_like(out, 5.0)
        S.page_attention(c, 0, wide[:, 1], at, max_len=max_len, max_new=max_new, out=again[:, :hq])
        torch.cuda.synchronize()
        assert torch.equal(again, out)                                  # the same call gives the same bits


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[1, 1, 1, 1], [2, 1, 6, 1], [90, 40, 70, 17]])
def test_rows_without_pages(counts, act, kind):
    """Pages that are missing in front (a window), in the middle, at the new tokens, and everywhere."""
    flush(f"case missing {counts} {act} {kind}")
    lens, P, hq, H, dh = [200, 90, 33, 70], 16, 8, 2, 64
    c, rows = paged(lens, counts, H, P, dh, kind, 21)
    c.table[0, :5] = -1
    c.table[1, 2], c.table[1, 3] = 1 << 20, -7
    c.table[2, 33 // P:] = -1
    c.table[3] = -1
    table = c.table.cpu()
    q = randn((sum(counts), hq, dh), DTYPES[act], 22)
    got = S.page_attention(c, 0, q.cuda(), starts(counts).cuda())
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, counts, P, act, dh ** -0.5,
          gone=lambda b, r: not 0 <= int(table[b, r // P]) < c.n_pages, some=edges)


@pytest.mark.parametrize("counts", [[4, 2, 3], [50, 20, 40]])
def test_lengths_out_of_range_and_tokens_beyond_the_table(counts):
    flush(f"case ranges {counts}")
    P, hq, H, dh = 16, 4, 2, 64
    lens = [-3, 60, 10]
    c, rows = paged([0, 60, 10], [64, 4, 54], H, P, dh, "int8", 23)
    assert c.max_seq == 64
    c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    q = randn((sum(counts), hq, dh), torch.bfloat16, 24)
    for L0 in (-3, 65, 1 << 30):
        c.len[0] = L0
        got = S.page_attention(c, 0, q.cuda(), starts(counts).cuda())
        torch.cuda.synchronize()
        check(got.double().cpu().numpy(), q.double().numpy(), rows[0], [L0, 60, 10], counts, P, "bf16", dh ** -0.5, cap=64, some=edges)
    # starts out of order or range: those sequences have no tokens
    out = torch.full((sum(counts), hq, dh), 5.0, dtype=torch.bfloat16, device="cuda")
    S.page_attention(c, 0, q.cuda(), torch.tensor([4, 2, -1, sum(counts) + 1], dtype=torch.int32).cuda(), out=out)
    torch.cuda.synchronize()
    assert out.eq(5).all()


@pytest.mark.parametrize("n", [6, 70])
@pytest.mark.parametrize("hq", [4, 16])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
def test_unseen_rows_reach_nothing(kind, hq, n):
    """Infinities and NaN in later tokens' rows and behind the last token: earlier tokens' outputs stay, bit for bit."""
    flush(f"case unseen {kind} {hq} {n}")
    lens, dh, P = [40, 0], 64, 16
    c, rows = paged(lens, [n, n], 2, P, dh, kind, 10, room=1)
    q = randn((2 * n, hq, dh), torch.bfloat16, 11).cuda()
    at = starts([n, n]).cuda()
    clean = S.page_attention(c, 0, q, at).view(2, n, hq, dh)
    for b in range(2):
        for i, what in ((3, math.nan), (n, math.inf), (n + 1, math.nan)):          # a later token, behind the last
            r = lens[b] + i
            page = int(c.table[b, r // P])
            if kind == "bf16":
                c.k[0, page, :, r % P] = what
                c.v[0, page, :, r % P, ::5] = what
                c.v[0, page, :, r % P, 1::5] = -math.inf
            elif kind == "e4m3":
                c.k.view(torch.uint8)[0, page, :, r % P] = 0x7f                     # NaN codes
                c.v.view(torch.uint8)[0, page, :, r % P] = 0x7f
        if kind == "int8":                                                          # a page of later tokens only
            page = int(c.table[b, (lens[b] + n - 1) // P])
            c.k_scale[0, page] = math.nan
            c.v_scale[0, page] = math.inf
    got = S.page_attention(c, 0, q, at).view(2, n, hq, dh)
    torch.cuda.synchronize()
    for b in range(2):
        first = 3 if kind != "int8" else max(0, (lens[b] + n - 1) // P * P - lens[b])
        assert torch.equal(got[b, :first], clean[b, :first]), b
        assert torch.isnan(got[b, first:]).any(-1).all(), b


@pytest.mark.parametrize("n", [3, 40])
def test_visible_infinities_stay_in_their_dimensions(n):
    flush(f"case visible infinities {n}")
    c, rows = paged([10], [n], 1, 16, 64, "bf16", 12)
    q = randn((n, 2, 64), torch.bfloat16, 13).cuda()
    at = starts([n]).cuda()
    clean = S.page_attention(c, 0, q, at)
    v = lambda r: c.v[0, int(c.table[0, r // 16]), 0, r % 16]          # noqa: E731
    v(11)[3], v(11)[4], v(11)[5] = math.inf, -math.inf, math.nan
    v(10)[4] = math.inf
    v(6)[8] = math.nan                                                  # a cached row
    got = S.page_attention(c, 0, q, at).float()
    torch.cuda.synchronize()
    # token 0 sees row 10, later ones row 11 too
    assert torch.isnan(got[:, :, 8]).all() and not torch.isfinite(got[0, :, 4]).any()
    assert not torch.isfinite(got[1:, :, 3]).any() and torch.isnan(got[1:, :, 4:6]).all()
    assert torch.equal(got[0, :, [3, 5]], clean[0, :, [3, 5]].float())
    rest = [d for d in range(64) if d not in (3, 4, 5, 8)]
    assert torch.equal(got[:, :, rest], clean.float()[:, :, rest])


@pytest.mark.parametrize("n", [2, 50])
def test_large_scores_and_one_step_rises(n):
    """Scores that grow along the cache by far more than one power of two per step, and a scale of its own."""
    flush(f"case rising scores {n}")
    c, rows = paged([700], [n], 1, 32, 64, "bf16", 14)
    ramp = torch.linspace(0, 1, c.max_seq)[:, None] * torch.ones(64)
    c.k[0, c.table[0].long(), 0] = ramp.view(-1, 32, 64).to(torch.bfloat16).cuda()
    rows[0][0][0] = ramp.to(torch.bfloat16).double().numpy()[:, None]
    q = torch.full((n, 2, 64), 1.0, dtype=torch.bfloat16)
    q[1::2] = -1.0
    got = S.page_attention(c, 0, q.cuda(), starts([n]).cuda(), scale=30.0)
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], [700], [n], 32, "bf16", 30.0, some=edges)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("dh", [64, 128])
def test_every_block_of_query_rows(dh, kind, act):
    """1, 2, 3 .. 4, 5 .. 8 and more tiles of 16 query rows, in one chunk and in several."""
    flush(f"case blocks {dh} {kind} {act}")
    for n, hq, lens, P in ((3, 4, [70, 1], 16), (5, 6, [33, 400], 32), (9, 6, [90, 700], 64), (13, 8, [5, 311], 128), (23, 8, [64, 190], 16),
                           (60, 5, [3, 250], 64)):
        c, rows = paged(lens, [n, n], 1, P, dh, kind, n)
        q = randn((2 * n, hq, dh), DTYPES[act], 50 + n)
        got = S.page_attention(c, 0, q.cuda(), starts([n, n]).cuda())
        torch.cuda.synchronize()
        check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, [n, n], P, act, dh ** -0.5, some=edges)


@pytest.mark.parametrize("kind", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed", "zeros"])
@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_scales_of_any_size(order, kind, act):
    """Values that grow or shrink by 40 powers of two along the cache, or are nothing but zeros."""
    flush(f"case scales {kind} {order} {act}")
    lens, n, hq, dh, P = [500, 130], 12, 8, 64, 16
    c, rows = paged(lens, [n, n], 1, P, dh, kind, 15)
    J = c.table.shape[1]
    x = torch.linspace(-20, 20, J)
    if order == "mixed":
        x = x[torch.randperm(J, generator=gen(16))]
    f = torch.zeros(J) if order == "zeros" else torch.exp2((x if order != "falling" else -x).round())
    for b in range(2):
        for j in range(J):
            page = int(c.table[b, j])
            if page < 0:
                continue
            if kind == "bf16":
                c.v[0, page] *= f[j].item()
            else:
                c.v_scale[0, page] *= f[j].item()
            rows[0][b][1][j * P:(j + 1) * P] *= f[j].item()
    for m in (1, n):
        q = randn((2 * m, hq, dh), DTYPES[act], 17)
        got = S.page_attention(c, 0, q.cuda(), starts([m, m]).cuda())
        torch.cuda.synchronize()
        check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, [m, m], P, act, dh ** -0.5)
        if order == "zeros":
            assert not got.any()


@pytest.mark.parametrize("n", [1, 20])
def test_visible_scales_that_are_not_finite(n):
    """A cached page whose scale is infinite or NaN: its sequence's outputs are not finite, and others' stay what they are."""
    flush(f"case scales not finite {n}")
    c, rows = paged([100, 100], [n, n], 1, 32, 64, "int8", 18)
    q = randn((2 * n, 8, 64), torch.bfloat16, 19).cuda()
    at = starts([n, n]).cuda()
    clean = S.page_attention(c, 0, q, at)
    for what in (math.inf, math.nan):
        c.v_scale[0, int(c.table[1, 1])] = what
        got = S.page_attention(c, 0, q, at)
        torch.cuda.synchronize()
        assert torch.equal(got[:n], clean[:n]) and not torch.isfinite(got[n:]).any()


def test_two_calls_at_once():
    """Two caches on two streams, a workspace of each call's own: what each gives alone."""
    flush("case two streams")
    runs = []
    for k in range(2):
        c, _ = paged([1500, 700, 3], [20, 1, 90], 2, 64, 128, "int8", 40 + k)
        runs.append((c, randn((111, 8, 128), torch.bfloat16, 50 + k).cuda(), torch.cuda.Stream()))
    at = starts([20, 1, 90]).cuda()
    alone = [S.page_attention(c, 0, q, at) for c, q, _ in runs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [S.page_attention(c, 0, q, at, stream=s.cuda_stream) for c, q, s in runs]
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, alone))
