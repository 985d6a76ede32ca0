"""Scores over rows of many logits that lie in one piece, whose sums a thread cannot hold in float32.

Tolerance, as in test_gpu_logprob, but for threads that add at most 512 terms before they meet in float64: arguments 2^-17; up to 32 shifts to a
new maximum, each by a factor that is off by 2^-22: 2^-17; exp2 and the factor in float64's place 2 x 2^-22; sums (512 + 6) 2^-24. So
e = 2^-16 + 2^-21 + 518 x 2^-24 for log2 s, whatever the row's length; a log probability b: ln 2 (e + 2^-23 |b|) + 2^-24 |b|; an entropy h:
e (1 + 2 h) + 2^-24 h."""
import math

import pytest
import torch

from paper_2609_29499_amd import session as S
from tests.seq_case import DTYPES, flush, gen

pytestmark = pytest.mark.gpu
E = 2.0 ** -16 + 2.0 ** -21 + 518 * 2.0 ** -24


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V,R,top", [(1 << 24, 512, 0), (1 << 24, 512, 3), ((1 << 20) + 77, 530, 32), (1 << 24, 3, 5), (32 * 4096 + 1, 600, 1), (64 * 4096, 600, 2)])
def test_long_rows(V, R, top, kind):
    """Rows that rise and fall by little and by much, noise of three sizes, one large logit among equal ones, a start of nothing."""
    flush(f"case long rows {V} {R} {top} {kind}")
    i = torch.arange(V, device="cuda")
    noise = torch.randn(V, generator=gen(V)).cuda()
    few = [i * (3.0 / V), i * (-3.0 / V), i * (4000.0 / V), i * (-400.0 / V), noise * 0.03, noise * 2.5, noise * 300.0, torch.where(i == 5, 0.0, -0.1),
           torch.where(i < V - 300, -math.inf, noise), torch.where(i < V // 2, noise, noise + 800.0)]
    few = torch.stack([r.float() for r in few]).to(DTYPES[kind])
    x = few.repeat(-(-R // len(few)), 1)[:R]
    n = min(R, len(few))
    tokens = torch.tensor([(7, V - 1, V // 2, V // 3)[k % 4] for k in range(R)], dtype=torch.int32, device="cuda")
    got = S.token_logprobs(x, tokens, top)
    for r in range(n):
        y = few[r].double()
        t = int(tokens[r])
        lps = torch.log_softmax(y, -1)
        p = lps.exp()
        h = -float(torch.where(p > 0, p * lps, 0.0).sum())
        lp = float(lps[t])
        near = lambda a, b: a == b if not math.isfinite(b) else abs(a - b) <= math.log(2) * (E + 2.0 ** -23 * abs(b)) + 2.0 ** -24 * abs(b)       # noqa: E731
        assert near(float(got.logprob[r]), lp), (r, float(got.logprob[r]), lp)
        assert abs(float(got.entropy[r]) - h) <= E * (1 + 2 * h) + 2.0 ** -24 * h, (r, float(got.entropy[r]), h)
        assert int(got.rank[r]) == int((y > y[t]).sum()) + int((y[:t] == y[t]).sum()), r
        if top:
            best = torch.sort(y, descending=True, stable=True).indices[:top]
            assert torch.equal(got.top_ids[r].long(), best), r
            assert all(near(float(a), float(b)) for a, b in zip(got.top_logprobs[r], lps[best])), r
    later = torch.arange(R, device="cuda") >= n
    for a in got[:5]:                   # rows repeat, but for their tokens
        if a is got.logprob or a is got.rank:
            continue
        assert torch.equal(a[later], a[(torch.arange(R, device="cuda") % len(few))[later]])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0, 3])
def test_more_rows_than_a_grid_has(top, kind):
    """A workgroup that takes more than one row."""
    R, V = 140001, 40
    flush(f"case many rows {top} {kind}")
    x = (torch.randn((R, V), generator=gen(4)) * 2).to(DTYPES[kind]).cuda()
    tokens = torch.randint(-1, V, (R,), generator=gen(5)).to(torch.int32).cuda()
    start = torch.tensor([0, 65535, 65537, R], dtype=torch.int32, device="cuda")
    got = S.token_logprobs(x, tokens, top, start=start)
    y = x.double()
    lps = torch.log_softmax(y, -1)
    there, at = tokens >= 0, tokens.clamp(min=0).long()[:, None]
    lp = torch.where(there, lps.gather(1, at)[:, 0], 0.0)
    near = lambda a, b: bool(((a.double() - b).abs() <= math.log(2) * (E + 2.0 ** -23 * b.abs()) + 2.0 ** -24 * b.abs()).all())       # noqa: E731
    assert near(got.logprob, lp)
    h = -(lps.exp() * lps).sum(-1)
    assert ((got.entropy.double() - h).abs() <= E * (1 + 2 * h) + 2.0 ** -24 * h).all()
    yt, ids = y.gather(1, at), torch.arange(V, device="cuda")
    assert torch.equal(got.rank.long(), torch.where(there, ((y > yt) | ((y == yt) & (ids < at))).sum(-1), -1))
    if top:
        best = torch.sort(y, dim=-1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(got.top_ids.long(), best) and near(got.top_logprobs, lps.gather(1, best))
    for i, (a, b) in enumerate(zip(start.tolist(), start.tolist()[1:])):
        assert near(got.mean[i], lp[a:b][there[a:b]].mean())
