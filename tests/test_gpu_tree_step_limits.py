"""A plan's step over drafted tokens where it ends and how it samples: every sequence's answer is the oracle's verification of
the step's own logits, over the nodes that fit the cache; its rows are the accepted path's."""
import pytest
import torch

import synth
from oracle import tree as O
from paper_2609_29499_amd import session as S
from synth.configs import Shape
from tests.seq_case import flush, gen, random_parents
from tests.test_gpu_tree_step import fill, plan_of

pytestmark = pytest.mark.gpu

SH = Shape(2, 512, 8, 2, 64, 1536, vocab=97)


def drafts(Bn, T, V, seed, chain_logits):
    """Tokens, u, and with chain_logits the distributions they are drawn from."""
    g = gen(seed)
    tokens = torch.randint(0, V, (Bn, T), generator=g).to(torch.int32)
    u = torch.rand((Bn, T), generator=g)
    u[:, 1::2] *= 0.05                                   # (drafts of an untrained plan are seldom taken otherwise)
    dl = torch.randn((Bn, T - 1, V), generator=g) if chain_logits else None
    return tokens, u, dl


def expect(logits, tokens, u, parent, dl, room, temperature):
    """(ids, path) of one sequence whose first `room` nodes fit."""
    T = min(room, len(tokens))
    if T < 1 or (parent is not None and parent[0] != -1):
        return [], []
    return O.verify(logits[:T], tokens[:T], None if u is None else u[:T], None if parent is None else parent[:T],
                    None if dl is None else dl[:T - 1], temperature)


def cache_of(plan, kind, lens, max_seq, seed):
    """A filled cache with these lengths, some of which may be out of range."""
    c = fill(plan, SH, kind, [max(0, min(x, max_seq)) for x in lens], max_seq, seed)[0]
    c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    return c


def rows_of(cache, max_seq):
    return [S.seq_read(cache, l, max_seq, dtype=torch.float32) for l in range(SH.n_layers)]


def run(plan, kind, seed, tokens, u, parent, dl, temperature, lens, max_seq):
    """One step against the oracle; returns the cache, n and the drafts accepted."""
    Bn, T = tokens.shape
    cache, twin = (cache_of(plan, kind, lens, max_seq, seed) for _ in range(2))
    before = rows_of(cache, max_seq)
    sh = SH
    table, scales = synth.embedding(sh)
    emb, sc = torch.from_numpy(table).cuda(), torch.from_numpy(scales).cuda()
    scratch = (torch.empty((Bn, T, sh.d_model), device="cuda"), torch.empty((Bn, T, sh.vocab), device="cuda"))
    d = lambda x: None if x is None else x.cuda()  # noqa: E731
    ids, path, n = plan.tree_step(emb, sc, tokens.cuda(), cache, u=d(u), parent=d(parent), draft_logits=d(dl),
                                  temperature=temperature, scratch=scratch)
    torch.cuda.synchronize()
    lg = scratch[1].double().cpu().numpy()
    after = cache.len.tolist()
    accepted = 0
    for b in range(Bn):
        room = max_seq - lens[b] if 0 <= lens[b] <= max_seq else 0
        wi, wp = expect(lg[b], tokens[b].tolist(), None if u is None else u[b].double().numpy(),
                        None if parent is None else parent[b].tolist(), None if dl is None else dl[b].double().numpy(), room, temperature)
        assert n[b].item() == len(wi), (b, n[b].item(), wi)
        assert ids[b].tolist() == wi + [-1] * (T - len(wi)) and path[b].tolist() == wp + [-1] * (T - len(wp)), b
        assert after[b] == lens[b] + len(wi)             # node 0 has a row, and every emitted token but the last
        accepted += max(len(wi) - 1, 0)
    # rows before the old lengths are what they were, those behind them the path's nodes' as the same layers append them
    plan.tree_forward(scratch[0], twin, d(parent))
    rows, nodes = rows_of(cache, max_seq), rows_of(twin, max_seq)
    for l in range(sh.n_layers):
        for k in range(2):
            for b in range(Bn):
                L = max(0, min(lens[b], max_seq))
                assert torch.equal(rows[l][k][b, :, :L], before[l][k][b, :, :L])
                at = [L + t for t in path[b].tolist() if t >= 0]
                assert torch.equal(rows[l][k][b, :, L:L + len(at)], nodes[l][k][b, :, at])
    return cache, n.tolist(), accepted


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("tree,draft,temperature", [(True, False, 0.7), (False, False, 1.3), (False, True, 0.9), (True, False, 0.0)])
def test_step_samples_what_the_oracle_does(kind, tree, draft, temperature):
    flush(f"case step samples {kind} {tree} {draft} {temperature}")
    lens, T, max_seq = [20, 0, 33], 6, 64
    store, fn, lm, plan = plan_of(SH, None, 3 * T, max_seq)
    accepted = 0
    for seed in range(4):
        tokens, u, dl = drafts(3, T, SH.vocab, 80 + seed, draft)
        parent = random_parents(3, T, seed) if tree else None
        accepted += run(plan, kind, seed, tokens, u if temperature else None, parent, dl, temperature, lens, max_seq)[2]
    flush(f"   accepted {accepted}")
    assert accepted > 0 or temperature == 0 or tree


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("tree,draft,temperature", [(True, False, 0.8), (False, False, 0.8), (False, True, 0.8), (False, False, 0.0)])
def test_sequences_at_the_end_of_the_cache(kind, tree, draft, temperature):
    """Three rows left, one, none, a length out of range, all there, and a sequence whose nodes are all absent: nodes that
    do not fit are not accepted, and a sequence whose node 0 is absent emits nothing and stays as it is."""
    flush(f"case step ends {kind} {tree} {draft} {temperature}")
    max_seq, T = 48, 6
    lens = [max_seq - 3, max_seq - 1, max_seq, -1, 10, max_seq + 5, 7]
    Bn = len(lens)
    store, fn, lm, plan = plan_of(SH, None, Bn * T, max_seq)
    ended = 0
    for seed in range(6):
        tokens, u, dl = drafts(Bn, T, SH.vocab, 90 + seed, draft)
        u[:, 1:] = 0.0                                   # (every draft with a share is taken: paths run into the end)
        parent = random_parents(Bn, T, seed, absent=False) if tree else None
        if tree:
            parent[6] = -2
        cache, n, _ = run(plan, kind, seed, tokens, u if temperature else None, parent, dl, temperature, lens, max_seq)
        assert n[2] == n[3] == n[5] == 0 and n[1] == 1 and (n[6] == 0) == tree
        ended += n[0] == 3
        k = cache.k.view(torch.uint8)[:, [2, 3, 5]].clone()
        again = plan_step_again(plan, cache, Bn, T)
        assert again[2][[2, 3, 5]].tolist() == [0, 0, 0] and torch.equal(cache.k.view(torch.uint8)[:, [2, 3, 5]], k)
    assert ended > 0 or temperature == 0 or tree


def plan_step_again(plan, cache, Bn, T):
    """Greedy steps from where the cache is, replayed from a graph: sequences at their end stay there."""
    table, scales = synth.embedding(SH)
    emb, sc = torch.from_numpy(table).cuda(), torch.from_numpy(scales).cuda()
    tokens = torch.zeros((Bn, T), dtype=torch.int32, device="cuda")
    ws = plan.tree_workspace(cache, T)
    scratch = (torch.empty((Bn, T, SH.d_model), device="cuda"), torch.empty((Bn, T, SH.vocab), device="cuda"))
    out = tuple(torch.empty(s, dtype=torch.int32, device="cuda") for s in ((Bn, T), (Bn, T), (Bn,)))
    keep = cache.len.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan.tree_step(emb, sc, tokens, cache, out=out, scratch=scratch, workspace=ws)
    side.synchronize()
    cache.len.copy_(keep)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        plan.tree_step(emb, sc, tokens, cache, out=out, scratch=scratch, workspace=ws)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
    return [t.cpu() for t in out]
