"""Verification of drafted tokens against the float64 oracle: whole numbers, so equal. The random numbers
are drawn once; both sides' sums are in 64 bits, so that a draw on a border (within 10^-13 of it) does not occur."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2609_29499_amd import session as S
from tests.seq_case import flush, gen, random_parents

pytestmark = pytest.mark.gpu


def inputs(Bn, T, V, seed, tree, draft, temperature):
    g = gen(seed)
    logits = torch.randn((Bn, T, V), generator=g) * 2.5
    if temperature == 0:
        logits = logits.to(torch.bfloat16).float()                  # ties of the largest logit
    parent = random_parents(Bn, T, seed) if tree else None
    dl = logits[:, :T - 1] + torch.randn((Bn, T - 1, V), generator=g) * 0.5 if draft else None
    u = torch.rand((Bn, T), generator=g)
    tokens = torch.zeros((Bn, T), dtype=torch.int32)
    src = dl if draft else logits
    for b in range(Bn):
        for t in range(1, T):
            p = t - 1 if parent is None else max(0, min(int(parent[b, t]), t - 1))
            row = src[b, p] / max(temperature, 0.3)
            pick = int(torch.multinomial(torch.softmax(row.double(), -1), 1, generator=g))
            tokens[b, t] = int(src[b, p].argmax()) if t % 3 == 1 else pick
    return logits, tokens, u, parent, dl


def run(logits, tokens, u, parent, dl, temperature, **kw):
    d = lambda x: None if x is None else x.cuda()  # noqa: E731
    ids, path, n = S.verify(d(logits), d(tokens), d(u), d(parent), d(dl), temperature, **kw)
    torch.cuda.synchronize()
    return ids.cpu().numpy(), path.cpu().numpy(), n.cpu().numpy()


def check(got, logits, tokens, u, parent, dl, temperature):
    ids, path, n = got
    Bn, T, _ = logits.shape
    for b in range(Bn):
        wi, wp = O.verify(logits[b].double().numpy(), tokens[b].tolist(), None if u is None else u[b].double().numpy(),
                          None if parent is None else parent[b].tolist(), None if dl is None else dl[b].double().numpy(), temperature)
        assert n[b] == len(wi) == len(wp)
        assert ids[b].tolist() == wi + [-1] * (T - len(wi)), b
        assert path[b].tolist() == wp + [-1] * (T - len(wp)), b


CASES = [
    # batch, T, vocab, tree, draft, temperature
    (1, 1, 1, False, False, 1.0), (3, 1, 2, False, False, 0.7), (2, 1, 128256, False, False, 0.8),
    (4, 5, 7, True, False, 1.0), (3, 64, 1000, True, False, 1.3), (5, 9, 4096, True, False, 0.6),
    (3, 12, 4097, False, False, 1.0), (2, 6, 50001, True, False, 0.3),
    (4, 5, 7, False, True, 1.0), (3, 9, 8192, False, True, 0.7), (2, 64, 301, False, True, 1.0),
    (1, 1, 333, False, True, 1.0), (2, 4, 20000, False, True, 0.9),
    (4, 8, 40, True, False, 0.0), (3, 20, 9000, False, False, 0.0), (2, 5, 12, False, True, 0.0),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_verify(case):
    Bn, T, V, tree, draft, temp = CASES[case]
    flush(f"case verify {CASES[case]}")
    x = inputs(Bn, T, V, case, tree, draft and T > 1, temp)
    if draft and T == 1:
        x = x[:4] + (torch.zeros((Bn, 0, V)),)
    check(run(*x, temp), *x[:4], None if T == 1 else x[4], temp)


def test_many_draws_of_a_small_vocabulary():
    """Every path through small trees: 256 sequences with tokens drawn at random, twice the same among siblings."""
    flush("case draws")
    for seed, draft in ((1, False), (2, True)):
        g = gen(seed)
        Bn, T, V = 256, 7, 4
        logits = torch.randn((Bn, T, V), generator=g)
        tokens = torch.randint(-1, V + 1, (Bn, T), generator=g).to(torch.int32)      # (outside the vocabulary too)
        u = torch.rand((Bn, T), generator=g)
        parent = None if draft else random_parents(Bn, T, seed)
        dl = torch.randn((Bn, T - 1, V), generator=g) if draft else None
        check(run(logits, tokens, u, parent, dl, 0.9), logits, tokens, u, parent, dl, 0.9)


def test_drawn_tokens_follow_the_target():
    """4096 draws over a fine grid of u: the counts are the probabilities, exactly up to the grid."""
    flush("case frequencies")
    V, n = 9, 256
    logits = torch.randn((1, 1, V), generator=gen(5)).repeat(n, 1, 1)
    counts = np.zeros(V)
    for k in range(16):
        u = ((torch.arange(n) * 16 + k).double() + 0.5) / (16 * n)
        ids, _, _ = run(logits, torch.zeros((n, 1), dtype=torch.int32), u.float()[:, None], None, None, 1.0)
        counts += np.bincount(ids[:, 0], minlength=V)
    p = O.softmax(logits[0, 0].double().numpy(), 1.0)
    assert np.all(np.abs(counts / (16 * n) - p) <= 1.5 / (16 * n))


def test_masked_and_degenerate_rows():
    """-inf and NaN logits, +inf, rows without anything, u at its ends, equal draft and target."""
    flush("case degenerate")
    V = 5000
    logits = torch.randn((6, 3, V), generator=gen(6))
    logits[0, 0, :4990] = -math.inf
    logits[1, 0] = -math.inf
    logits[1, 0, 4321] = torch.finfo(torch.float32).min            # the type's lowest value alone
    logits[2, 0, 7], logits[2, 0, 4500] = math.inf, math.inf
    logits[3, 0] = math.nan
    logits[4, 0, ::2] = math.nan
    logits[5, 0] = 0.0
    u = torch.full((6, 3), 0.999999940395355)                        # 1 - 2^-24
    u[4], u[2] = 0.0, 0.5
    tokens = torch.tensor([[0, 4999, 1], [0, 4321, 2], [0, 8, 3], [0, 5, 5], [0, 1, 1], [0, 4999, 4998]], dtype=torch.int32)
    for temp in (1.0, 0.5, 0.0):
        for dl in (None, torch.randn((6, 2, V), generator=gen(7)), logits[:, :2].clone()):
            x = (logits, tokens, u, None, dl)
            check(run(*x, temp), *x, temp)


def test_a_vocabulary_with_equal_shares():
    """Every border of 32768 equal shares, from both sides of u: the lowest token whose cumulative share exceeds it."""
    flush("case borders")
    V = 32768
    Bn = 64
    k = torch.arange(Bn) * 512
    u = (k.double() / V).float()[:, None]
    ids, _, _ = run(torch.zeros((Bn, 1, V)), torch.zeros((Bn, 1), dtype=torch.int32), u, None, None, 1.0)
    assert ids[:, 0].tolist() == k.tolist()


@pytest.mark.parametrize("draft", [False, True])
def test_a_vocabulary_of_more_chunks_than_lanes(draft):
    flush(f"case wide vocabulary {draft}")
    V, T = 300001, 3
    g = gen(21)
    logits = torch.randn((3, T, V), generator=g)
    logits[1] *= 0.01                   # nearly even: the last token lies anywhere
    logits[2, :, :280000] = -math.inf
    dl = logits[:, :2] + torch.randn((3, 2, V), generator=g) if draft else None
    tokens = torch.tensor([[0, 5, 6], [0, 299999, 7], [0, 300000, 290000]], dtype=torch.int32)
    u = torch.tensor([[0.3, 0.9, 0.1], [0.97, 0.9, 0.2], [0.999, 0.0, 0.9]])
    check(run(logits, tokens, u, None, dl, 0.9), logits, tokens, u, None, dl, 0.9)
    check(run(logits, tokens, u, None, dl, 0.0), logits, tokens, u, None, dl, 0.0)


def test_ends_of_the_temperature():
    """The coldest takes the largest logit whatever u; the hottest gives every finite logit the same share."""
    flush("case temperatures")
    V = 6000
    logits = torch.randn((4, 1, V), generator=gen(22)) * 1e30
    logits[:, :, 100:200] = -math.inf
    logits[1, 0, 5999] = torch.finfo(torch.float32).max
    u = torch.tensor([[0.0], [0.5], [0.25], [0.999]])
    tokens = torch.zeros((4, 1), dtype=torch.int32)
    ids, _, _ = run(logits, tokens, u, None, None, 1e-30)
    assert ids[:, 0].tolist() == logits[:, 0].argmax(-1).tolist()
    flat = logits / 1e30
    ids, _, _ = run(flat, tokens, u, None, None, 1e30)
    ok = torch.cat([torch.arange(100), torch.arange(200, V)])
    want = [int(ok[int(x * 5900)]) for x in u[:, 0].double().tolist()]
    # differences of 1 weigh 1e-30 at this temperature: shares are equal to all of 64 bits; u on a border takes the token behind it
    assert ids[:, 0].tolist() == want


def test_two_calls_at_once():
    """Calls on two streams with a workspace each, a raw stream among them, give what they give alone."""
    flush("case two streams")
    a, b = (inputs(4, 9, 20000, 30 + k, False, True, 0.8) for k in range(2))
    alone = [run(*x, 0.8) for x in (a, b)]
    dev = [[None if t is None else t.cuda() for t in x] for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [S.verify(*x, 0.8, stream=s.cuda_stream) for x, s in zip(dev, streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, alone):
            for p, q in zip(g, w):
                assert np.array_equal(p.cpu().numpy(), q)
