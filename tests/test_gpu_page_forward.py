"""A plan over packed tokens of several sequences in pages (tasp_page_forward): every token's output against the float64
oracle, and a run as a server does it: prompts in chunks, single tokens, scores of what comes out, the router's input."""
import numpy as np
import pytest
import torch

import synth
from oracle import reference as ref
from oracle import score as OS
from paper_2609_29499_amd import binding as B
from paper_2609_29499_amd import session as S
from synth import text as text_inputs
from synth.configs import Shape
from tests.helpers import assert_parity
from tests.page_case import starts, table_of
from tests.seq_case import DTYPES, flush, gen
from tests.test_gpu_tree_step import plan_of

pytestmark = pytest.mark.gpu


def pool(plan, sh, lens, counts, P, kind, seed, room=0):
    pages = [-(-(n + c) // P) + room for n, c in zip(lens, counts)]
    table, n = table_of([max(1, p) for p in pages], max(pages + [1]), seed)
    cache = S.PageCache.empty(sh.n_layers, n, sh.n_kv_heads, P, sh.head_dim, len(lens), table.shape[1], DTYPES[kind])
    cache.table.copy_(table)
    plan.page_bind(cache)
    return cache


def fill(cache, sh, lens, seed):
    """Synthetic rows of every sequence, written by the append without rotation; returns the oracle's caches."""
    g = gen(seed)
    at = starts(lens).cuda()
    caches = []
    for l in range(sh.n_layers):
        k, v = (torch.randn((max(1, sum(lens)), sh.n_kv_heads, sh.head_dim), generator=g) for _ in range(2))
        if sum(lens):
            S.page_append(cache, l, None, k.cuda(), v.cuda(), at)
        gk, gv = S.page_read(cache, l, cache.max_seq, dtype=torch.float32)
        caches.append((gk.double().cpu().numpy(), gv.double().cpu().numpy()))
    cache.len.copy_(torch.tensor(lens, dtype=torch.int32))
    return caches


CASES = [
    # shape, mask kept shares, lens, counts (None: one each), rows of a page, cache, shared store
    (Shape(2, 512, 8, 2, 64, 1536), True, [20, 0, 33], [5, 12, 1], 16, "bf16", False),
    (Shape(1, 512, 16, 4, 64, 768), True, [129, 64], [40, 1], 32, "bf16", False),
    (Shape(1, 1024, 8, 1, 128, 512), False, [300, 2], [9, 70], 64, "bf16", False),
    (Shape(2, 512, 8, 2, 64, 1536, vocab=300), True, [40, 900, 0], None, 16, "bf16", False),
    (Shape(1, 512, 8, 2, 64, 1536, vocab=517), True, [17, 90], [7, 3], 128, "bf16", True),
    (Shape(1, 512, 16, 4, 64, 768), True, [47, 64, 80], [1, 16, 20], 16, "int8", False),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_page_forward(case):
    sh, masked, lens, counts, P, kind, shared = CASES[case]
    flush(f"case page forward {CASES[case]}")
    rng = np.random.default_rng(case)
    mask = None
    if masked:                          # uneven groups: the first loses heads, another may go altogether
        q = np.ones((sh.n_layers, sh.n_q_heads), np.uint8)
        q[:, 0] = 0
        q[0, 1] = 0
        q[0, -sh.group_size:] = sh.n_kv_heads < 3
        f = np.ones((sh.n_layers, sh.d_ffn), np.uint8)
        f[:, 16 * rng.permutation(sh.d_ffn // 16)[:, None] + np.arange(16)] = (rng.random((sh.d_ffn // 16, 1)) < 0.7)
        mask = (q, None, f)
    n = [1] * len(lens) if counts is None else counts
    front, behind = (0, 0) if counts is None else (2, 1)               # tokens of no sequence
    N = front + sum(n) + behind
    store, fn, lm, plan = plan_of(sh, mask, N, 64, shared)
    cache = pool(plan, sh, lens, n, P, kind, case)
    caches = fill(cache, sh, lens, case)
    x = synth.activations(N, sh.d_model, 3)
    x[:front] = np.nan
    xd = torch.from_numpy(x).cuda()
    out = plan.page_forward(xd, cache, None if counts is None else starts(n, front).cuda())
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    closed = ref.close_mask(*(mask if mask is not None else synth.all_kept_mask(sh)), sh.group_size)
    t0 = front
    for b, (L, c) in enumerate(zip(lens, n)):
        own = [(k[b].copy(), v[b].copy()) for k, v in caches]
        want = ref.prefill_stack(lambda l: store[l], closed, x[t0:t0 + c], own, L, sh, fn, lm, kv_store=ref.bf16_store)
        # 8 bits: new rows are a quarter of a code off on average (BF16 in the oracle), older ones once more where a scale rises;
        # of scores and values 1 / 127 / 4 a row and all, which a dozen rows and the residual stream average out
        assert_parity(got[t0:t0 + c], want, max_rel=1e-2 if kind == "bf16" else 4e-2, sum_rel=2e-3 if kind == "bf16" else 1e-2, what=f"seq {b}")
        t0 += c
    assert cache.len.tolist() == lens
    S.page_advance(cache, N, None if counts is None else starts(n, front).cuda())
    assert cache.len.tolist() == [a + b for a, b in zip(lens, n)]


def test_chunks_single_tokens_scores_and_the_router():
    """Three conversations through one pool: prompts in chunks beside single tokens, a captured decoding step replayed,
    every token scored, the prompts' mean log probabilities handed to the router."""
    flush("case serving run")
    sh = Shape(2, 512, 8, 2, 64, 768, vocab=400)
    store, fn, lm, plan = plan_of(sh, None, 64, 256)
    table, scales = synth.embedding(sh)
    emb = torch.from_numpy(table).float().cuda() * torch.from_numpy(scales).cuda()[:, None]
    prompts = [synth.prompt_ids(n, sh.vocab, seed=i) for i, n in enumerate((45, 20, 3))]
    cache = pool(plan, sh, [0] * 3, [64] * 3, 16, "bf16", 5)
    closed = ref.close_mask(*synth.all_kept_mask(sh), sh.group_size)
    text = [p.tolist() for p in prompts]

    def oracle(b):
        x = (table.astype(np.float64) * scales.astype(np.float64)[:, None])[text[b]]
        own = [tuple(np.zeros((sh.n_kv_heads, 128, sh.head_dim)) for _ in range(2)) for _ in range(sh.n_layers)]
        return ref.prefill_stack(lambda l: store[l], closed, x, own, 0, sh, fn, lm, kv_store=ref.bf16_store)

    logits = [[] for _ in range(3)]
    # a chunk of the first prompt with the whole second; its rest beside single tokens of the second and the whole third
    sent = [0, 0, 0]
    for counts in ([30, 20, 0], [15, 0, 3]):
        ids = np.concatenate([text[b][sent[b]:sent[b] + c] for b, c in enumerate(counts)]).astype(np.int64)
        at = starts(counts).cuda()
        out = plan.page_forward(emb[torch.from_numpy(ids).cuda()], cache, at, max_len=45, max_new=30)
        S.page_advance(cache, len(ids), at)
        o = 0
        for b, c in enumerate(counts):
            logits[b].append(out[o:o + c])
            sent[b] += c
            o += c
    last = torch.stack([logits[b][-1][-1] if logits[b][-1].shape[0] else logits[b][0][-1] for b in range(3)])
    # decoding: one captured step, the highest token fed back on the device
    ids = S.token_logprobs(last, torch.zeros(3, dtype=torch.int32, device="cuda"), 1).top_ids[:, 0].clone()
    x = emb[ids.long()].contiguous()
    ws, wl = plan.page_workspace(cache, 3, 64, 1), S.token_logprobs_workspace(3, sh.vocab, 4)
    step_out = torch.empty((3, sh.vocab), device="cuda")

    def step():
        x.copy_(emb[ids.long()])
        plan.page_forward(x, cache, None, max_len=64, max_new=1, out=step_out, workspace=ws)
        sc = S.token_logprobs(step_out, ids, 4, workspace=wl)
        S.page_advance(cache, 3)
        ids.copy_(sc.top_ids[:, 0])
        return sc

    saved = [t.clone() for t in (cache.k, cache.v, cache.len, ids)]
    step()                              # (once outside of the capture, taken back)
    torch.cuda.synchronize()
    for t, o in zip((cache.k, cache.v, cache.len, ids), saved):
        t.copy_(o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sc = step()
    for _ in range(6):
        fed = ids.tolist()
        graph.replay()
        torch.cuda.synchronize()
        for b in range(3):
            text[b].append(fed[b])
            logits[b].append(step_out[b:b + 1].clone())
        want = S.token_logprobs(step_out, torch.tensor(fed, dtype=torch.int32, device="cuda"), 4)
        assert all(torch.equal(a, b) for a, b in zip(sc[:5], want[:5]))
    assert cache.len.tolist() == [45 + 6, 20 + 6, 3 + 6]
    got = [torch.cat(v) for v in logits]
    for b in range(3):
        assert_parity(got[b].double().cpu().numpy(), oracle(b), what=f"conversation {b}")
    # the prompts' scores: logits of each position against the next token
    rows = torch.cat([got[b][:len(prompts[b]) - 1] for b in range(3)])
    tokens = torch.tensor(np.concatenate([p[1:] for p in prompts]).astype(np.int32), device="cuda")
    at = starts([len(p) - 1 for p in prompts])
    sc = S.token_logprobs(rows, tokens, 2, start=at.cuda())
    torch.cuda.synchronize()
    lps = [OS.score(r, t)[0] for r, t in zip(rows.double().cpu().numpy(), tokens.tolist())]
    np.testing.assert_allclose(sc.mean.cpu().numpy(), OS.mean(lps, tokens.tolist(), sh.vocab, at.tolist()), rtol=2.0 ** -16)
    router = S.Router(text_inputs.router_weights(n_bins=64, proj_dim=16, hidden1=32, hidden2=16, n_tasks=3))
    words = torch.tensor(list(b"solve 2 + 2, then translate this"), dtype=torch.uint8, device="cuda")
    feats, _, _ = router.route(words, torch.tensor([0, 10, 20, words.numel()], dtype=torch.int32, device="cuda"), sc.mean)
    torch.cuda.synchronize()
    assert torch.equal(feats[:, 17], sc.mean)          # behind the projection and the length


def test_refusals():
    sh = Shape(1, 512, 8, 2, 64, 768)
    store, fn, lm, plan = plan_of(sh, None, 32, 64)
    cache = pool(plan, sh, [0, 0], [40, 40], 16, "int8", 1)
    x = torch.zeros((4, 512), device="cuda")
    at = starts([3, 1]).cuda()
    plan.page_forward(x, cache, at)
    for f, status in ((lambda: plan.page_forward(torch.zeros((33, 512), device="cuda"), cache, at), "TASP_ERR_SHAPE"),
                      (lambda: plan.page_forward(x, cache), "TASP_ERR_SHAPE"),
                      (lambda: plan.page_forward(x, cache, at, max_len=49), "TASP_ERR_SHAPE"),
                      (lambda: plan.page_forward(x, cache, at, max_new=0), "TASP_ERR_SHAPE"),
                      (lambda: plan.page_forward(x, cache, at, out=x), "TASP_ERR_INVALID_ARG")):
        with pytest.raises(B.TaspError) as e:
            f()
        assert B.STATUS[e.value.status] == status, e.value
    other = S.PageCache.empty(1, 4, 2, 16, 64, 2, 3)
    with pytest.raises(B.TaspError, match="belongs to plan"):
        plan.page_forward(x, other, at)
    with pytest.raises(B.TaspError) as e:
        plan.page_bind(S.PageCache.empty(1, 4, 1, 16, 64, 2, 3))
    assert B.STATUS[e.value.status] == "TASP_ERR_SHAPE"
    torch.cuda.synchronize()
