"""Scores of given tokens against the float64 oracle.

Tolerances. t = (x - m) c, c = log2(e) / temperature: the difference, the product and c itself are rounded, as is a shift to a new
maximum: 4 x 2^-24 |t|. Weighted by the terms 2^t, |t| is 32 at most (a mean of |t| under p is the entropy in bits less log2 s, and
log2 of the vocabulary bounds both): 2^-17. exp2 is off by 2^-22. A thread adds at most n = 16 ceil(V / 4096) terms in float32,
n 2^-24 of their sum, and its wave 6 more. So log2 s is off by e = 2^-17 + 2^-22 + (n + 6) 2^-24 at most, a log probability b by
ln 2 (e + 2^-23 |b|) (c's rounding once more) and its own 2^-24 |b|, the entropy h, whose terms t 2^t carry the same relative
errors, by e (1 + 2 h) and its own rounding."""
import math

import numpy as np
import pytest
import torch

from oracle import score as O
from paper_2609_29499_amd import session as S
from tests.seq_case import DTYPES, flush, gen

pytestmark = pytest.mark.gpu


def check(got, logits, tokens, temperature, n_top, start=None, rows=None):
    x = logits.double().cpu().numpy()
    R, V = x.shape
    e = 2.0 ** -17 + 2.0 ** -22 + (16 * -(-V // 4096) + 6) * 2.0 ** -24
    lps = []
    got = S.TokenLogprobs(*[None if t is None else t.cpu().double().numpy() for t in got])

    def near(a, b, extra=0.0):
        if not math.isfinite(b):
            return a == b
        return abs(a - b) <= math.log(2) * (e + 2.0 ** -23 * abs(b)) + 2.0 ** -24 * abs(b) + extra

    for r in range(R) if rows is None else rows:
        lp, h, rank, ids, tops = O.score(x[r], int(tokens[r]), temperature, n_top)
        assert near(got.logprob[r], lp), (r, got.logprob[r], lp)
        assert abs(got.entropy[r] - h) <= e * (1 + 2 * h) + 2.0 ** -24 * h, (r, got.entropy[r], h)
        assert got.rank[r] == rank, (r, got.rank[r], rank)
        assert got.top_ids[r].tolist() == ids, (r, got.top_ids[r], ids)
        assert all(near(a, b) for a, b in zip(got.top_logprobs[r], tops)), (r, got.top_logprobs[r], tops)
        lps.append(lp)
    if start is not None and rows is None:
        for a, b in zip(got.mean, O.mean(lps, tokens.tolist(), V, start.tolist())):
            assert near(a, b)


CASES = [
    # rows, vocab, n_top, logits, temperature
    (1, 1, 0, "f32", 1.0), (1, 1, 4, "f32", 1.0), (3, 2, 1, "bf16", 0.5), (7, 31, 32, "f32", 1.0), (2, 32, 32, "bf16", 1.0),
    (5, 4095, 20, "f32", 0.7), (5, 4096, 20, "f32", 1.0), (5, 4097, 5, "bf16", 1.3), (3, 32003, 32, "bf16", 1.0),
    (2, 128256, 20, "f32", 1.0), (1, 128256, 1, "f32", 0.25), (40, 9001, 0, "f32", 1.0), (3, 70001, 7, "f32", 100.0),
    (1030, 5003, 3, "f32", 1.0), (600, 8200, 16, "bf16", 1.0),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_scores(case):
    R, V, top, kind, temperature = CASES[case]
    flush(f"case scores {CASES[case]}")
    g = gen(case)
    x = (torch.randn((R, V), generator=g) * 3).to(DTYPES[kind])
    tokens = torch.randint(0, V, (R,), generator=g).to(torch.int32)
    tokens[::3] = x[::3].float().argmax(-1).to(torch.int32)
    if R > 4:
        tokens[3], tokens[4] = -1, V
    start = torch.tensor([0, R // 3, R // 3, R], dtype=torch.int32)
    got = S.token_logprobs(x.cuda(), tokens.cuda(), top, temperature, start.cuda())
    torch.cuda.synchronize()
    rows = None if R < 50 else list(range(0, R, R // 13)) + [R - 1]
    check(got, x, tokens, temperature, top, start, rows)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V,R", [(9000, 12), (5000, 700), (40, 3)])
def test_orders_and_ties(V, R, kind):
    """Rows that rise, fall, are constant, take few values, or have their largest values in one place: lists overflow, equal
    logits come by id."""
    flush(f"case orders {V} {R} {kind}")
    g = gen(V)
    rows = [torch.arange(V) * 1e-3, torch.arange(V).flip(0) * 1e-3, torch.full((V,), -7.0), torch.zeros(V),
            torch.randint(0, 3, (V,), generator=g).float(), torch.where(torch.arange(V) == V - 1, 50.0, -1.0),
            torch.where(torch.arange(V) < 40, 5.0, 1.0), torch.where(torch.arange(V) % 16 == 3, 2.0, -0.0),
            torch.where(torch.arange(V) >= V - 100, torch.arange(V) * 1.0, 0.0), -torch.zeros(V)]
    x = torch.stack([rows[i % len(rows)] for i in range(R)]).to(DTYPES[kind])
    tokens = torch.randint(0, V, (R,), generator=g).to(torch.int32)
    for top in (1, 3, 32):
        got = S.token_logprobs(x.cuda(), tokens.cuda(), top)
        again = S.token_logprobs(x.cuda(), tokens.cuda(), top)
        torch.cuda.synchronize()
        check(got, x, tokens, 1.0, top, rows=list(range(min(R, 10))) + [R - 1])
        assert all(torch.equal(a, b) for a, b in zip(got[:5], again[:5]))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("R", [1, 520])
def test_largest_logits_in_few_places(R, kind):
    """All large logits where one thread, one wave or one tile reads them, in both orders, and rows of one value but for these: lists
    that fill up again and again, for rows in one piece and in many."""
    flush(f"case few places {R} {kind}")
    V = 40000
    i = torch.arange(V)
    rows = [torch.where(i % 256 == 7, i / 64.0, -5.0), torch.where(i % 256 == 7, -i / 64.0, -900.0),
            torch.where((i // 4) % 256 < 8, i % 97 / 8.0, 0.0), torch.where(i // 4096 == 3, 2.0, 1.0), torch.where(i % 1024 == 9, 1.0, 0.0),
            torch.where(i > V - 50, 3.0, -1.0), (i // 3000).float(), -(i // 3000).float()]
    x = torch.stack([rows[k % len(rows)] for k in range(R)] if R > 1 else rows).to(DTYPES[kind])
    for k in range(len(rows)):
        one = x[k:k + 1] if R == 1 else x
        tokens = torch.randint(0, V, (one.shape[0],), generator=gen(k)).to(torch.int32)
        for top in (1, 5, 32):
            got = S.token_logprobs(one.cuda(), tokens.cuda(), top)
            torch.cuda.synchronize()
            check(got, one, tokens, 1.0, top, rows=None if R == 1 else range(len(rows)))
        if R > 1:
            break


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 6000])
def test_rows_with_infinities_and_nan(V, kind):
    flush(f"case infinities {V} {kind}")
    inf, nan = math.inf, math.nan
    x = torch.randn((9, V), generator=gen(3)).to(DTYPES[kind])
    x[0] = -inf                                        # no token at all
    x[1] = nan
    x[2, 1] = inf
    x[3, 0], x[3, V - 1] = inf, inf
    x[4, 1:] = -inf                                    # one token
    x[5, ::2] = nan
    x[6, ::2] = -inf
    x[7] = -inf
    x[7, V - 1], x[7, 2] = inf, nan
    x[8, 3] = 3e38
    tokens = torch.tensor([2, 0, 1, V - 1, 0, 1, 1, V - 1, 3], dtype=torch.int32)
    for tok in (tokens, torch.full((9,), 2, dtype=torch.int32)):
        got = S.token_logprobs(x.cuda(), tok.cuda(), 4)
        torch.cuda.synchronize()
        check(got, x, tok, 1.0, 4)


def test_temperatures_at_their_ends():
    flush("case temperatures")
    x = torch.randn((4, 3000), generator=gen(4))
    tokens = x.argmax(-1).to(torch.int32)
    tokens[1] = 5
    got = S.token_logprobs(x.cuda(), tokens.cuda(), 2, 1e30)
    torch.cuda.synchronize()
    check(got, x, tokens, 1e30, 2)
    got = S.token_logprobs(x.cuda(), tokens.cuda(), 2, 1e-30)
    torch.cuda.synchronize()
    assert got.logprob[0] == 0.0 and got.entropy[0] == 0.0 and got.logprob[1] < -1e28 and got.top_logprobs[:, 0].eq(0).all()
    assert torch.equal(got.top_ids[:, :2].cpu().long(), torch.topk(x, 2).indices)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_strided_and_misaligned_rows(kind):
    """Rows inside wider ones, from an odd element on."""
    flush(f"case strided {kind}")
    wide = torch.randn((6, 9001), generator=gen(5)).to(DTYPES[kind]).cuda()
    wide[:, 0] = math.nan
    wide[:, 8501:] = 1e30
    x = wide[:, 1:8501]
    tokens = torch.arange(6, dtype=torch.int32) * 100
    got = S.token_logprobs(x, tokens.cuda(), 5)
    torch.cuda.synchronize()
    check(got, x, tokens, 1.0, 5)


def test_means_feed_the_router_and_ragged_bounds():
    flush("case means")
    x = torch.randn((50, 300), generator=gen(6))
    tokens = torch.randint(0, 300, (50,), generator=gen(7)).to(torch.int32)
    tokens[10:13] = -1
    start = torch.tensor([-4, 3, 10, 13, 13, 40, 99], dtype=torch.int32)    # in front of the rows, padding only, empty, behind
    got = S.token_logprobs(x.cuda(), tokens.cuda(), 0, start=start.cuda())
    torch.cuda.synchronize()
    check(got, x, tokens, 1.0, 0, start)
    assert got.mean.shape == (6,) and got.mean[2] == 0 and got.mean[3] == 0
    down = S.token_logprobs(x.cuda(), tokens.cuda(), 0, start=torch.tensor([20, 10], dtype=torch.int32).cuda())
    assert down.mean.item() == 0.0


def test_logits_behind_32_bit_offsets():
    flush("case far rows")
    V, R = 128256, 17000                               # 2^31 logits and more
    x = torch.zeros((R, V), dtype=torch.bfloat16, device="cuda")
    x[R - 1, V - 1], x[R - 1, 7] = 9.0, 8.0
    tokens = torch.full((R,), V - 1, dtype=torch.int32, device="cuda")
    got = S.token_logprobs(x, tokens, 2)
    torch.cuda.synchronize()
    assert got.top_ids[R - 1].tolist() == [V - 1, 7] and got.top_ids[:R - 1].eq(torch.tensor([0, 1], device="cuda")).all()
    assert got.rank[R - 1] == 0 and got.rank[:R - 1].eq(V - 1).all()
    np.testing.assert_allclose(got.logprob[:R - 1].cpu().numpy(), -math.log(V), rtol=2.0 ** -20)


def test_captured_and_on_two_streams():
    """Calls replayed in a graph with new logits in the same memory, and two calls at once with a workspace each."""
    flush("case graph")
    x = torch.randn((6, 50000), generator=gen(8)).cuda()
    tokens = torch.randint(0, 50000, (6,), generator=gen(9)).to(torch.int32).cuda()
    start = torch.tensor([0, 2, 6], dtype=torch.int32).cuda()
    ws = S.token_logprobs_workspace(6, 50000, 20)
    S.token_logprobs(x, tokens, 20, start=start, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = S.token_logprobs(x, tokens, 20, start=start, workspace=ws)
    for k in range(4):
        x.copy_(torch.randn((6, 50000), generator=gen(20 + k)).cuda())
        graph.replay()
        torch.cuda.synchronize()
        want = S.token_logprobs(x, tokens, 20, start=start)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for k in range(4):
        got = []
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            got.append(S.token_logprobs(x, tokens, 20, start=start, stream=s.cuda_stream))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
