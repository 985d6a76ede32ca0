"""A plan's step over trees of drafted tokens (tasp_tree_forward, tasp_tree_step): every node's output against
the float64 oracle run along the node's own path, and whole runs against greedy decoding."""
import numpy as np
import pytest
import torch

import synth
from oracle import reference as ref
from oracle import tree as O
from paper_2609_29499_amd import binding as B
from paper_2609_29499_amd import session as S
from synth.configs import Shape
from tests.helpers import assert_parity
from tests.seq_case import DTYPES, flush, gen, random_parents

pytestmark = pytest.mark.gpu


def held(kind):
    """The oracle's cache store: rows as the cache holds them."""
    if kind == "bf16":
        return ref.bf16_store

    def store(a):
        top = np.abs(a).max(-1, keepdims=True)
        return np.round(a * 127.0 / np.where(top > 0, top, 1.0)) * (top / 127.0)
    return store


def plan_of(sh, mask, max_prefill, max_seq, shared=False):
    store = [synth.layer_weights(sh, l, 0, quant="group" if shared else "row") for l in range(sh.n_layers)]
    fn, lm = (synth.final_norm(sh), synth.lm_head(sh)) if sh.vocab else (None, None)
    desc = S.desc_from_shape(sh, max_batch=1, max_seq=max_seq, max_prefill=max_prefill)
    if shared:
        return store, fn, lm, S.Plan.shared(desc, S.GroupStore(store, fn, lm), mask)
    return store, fn, lm, S.Plan(desc, S.DeviceStore(store, fn, lm), mask)


def fill(plan, sh, kind, lens, max_seq, seed):
    """A typed cache with synthetic rows (written by the append, keys unrotated in both) and the oracle's caches."""
    cache = S.SeqCache.empty(sh.n_layers, len(lens), sh.n_kv_heads, max_seq, sh.head_dim, DTYPES[kind])
    n = max(max(lens), 1)
    g = gen(seed)
    caches = []
    for l in range(sh.n_layers):
        k, v = (torch.randn((len(lens), n, sh.n_kv_heads, sh.head_dim), generator=g) for _ in range(2))
        S.seq_append(cache, l, None, k.cuda(), v.cuda())
        gk, gv = S.seq_read(cache, l, max_seq, dtype=torch.float32)
        caches.append((gk.double().cpu().numpy(), gv.double().cpu().numpy()))
    cache.len.copy_(torch.tensor(lens, dtype=torch.int32))
    plan.seq_bind(cache)
    return cache, caches


CASES = [
    # shape, mask kept shares, lens, T, cache, shared store
    (Shape(2, 512, 8, 2, 64, 1536), True, [20, 0, 33], 5, "bf16", False),
    (Shape(1, 512, 16, 4, 64, 768), True, [129, 64], 16, "int8", False),
    (Shape(1, 1024, 8, 1, 128, 512), False, [300], 9, "bf16", False),
    (Shape(2, 512, 8, 2, 64, 1536, vocab=300), True, [40], 1, "int8", False),
    (Shape(1, 512, 8, 2, 64, 1536, vocab=517), True, [17, 90], 7, "bf16", True),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_tree_forward(case):
    sh, masked, lens, T, kind, shared = CASES[case]
    flush(f"case tree forward {CASES[case]}")
    rng = np.random.default_rng(case)
    mask = None
    if masked:                          # uneven groups: the first loses heads, another may go altogether
        q = np.ones((sh.n_layers, sh.n_q_heads), np.uint8)
        q[:, 0] = 0
        q[0, -sh.group_size:] = sh.n_kv_heads < 3
        f = np.ones((sh.n_layers, sh.d_ffn), np.uint8)
        f[:, 16 * rng.permutation(sh.d_ffn // 16)[:, None] + np.arange(16)] = (rng.random((sh.d_ffn // 16, 1)) < 0.7)
        mask = (q, None, f)
    max_seq = max(lens) + T + 3
    store, fn, lm, plan = plan_of(sh, mask, len(lens) * T, max_seq, shared)
    cache, caches = fill(plan, sh, kind, lens, max_seq, case)
    parent = random_parents(len(lens), T, case)
    x = synth.activations(len(lens) * T, sh.d_model, 3).reshape(len(lens), T, sh.d_model)
    out = plan.tree_forward(torch.from_numpy(x).cuda(), cache, parent.cuda())
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    closed = ref.close_mask(*(mask if mask is not None else synth.all_kept_mask(sh)), sh.group_size)
    for b in range(len(lens)):
        for t, line in enumerate(O.lines(parent[b].tolist(), T)):
            if line is None:
                continue
            own = [(k[b].copy(), v[b].copy()) for k, v in caches]
            want = ref.prefill_stack(lambda l: store[l], closed, x[b, line], own, lens[b], sh, fn, lm, kv_store=held(kind))
            # codes at a border may fall either way in 8 bits: one step of 1 / 127 in a node's own rows
            assert_parity(got[b, t], want[-1], sum_rel=2e-3 if kind == "bf16" else 5e-3, what=f"seq {b} node {t}")
    assert cache.len.tolist() == lens


def request(sh, T, n_new, seed=0):
    store, fn, lm, plan = plan_of(sh, None, max(T, 64), T + n_new + 80)
    table, scales = synth.embedding(sh)
    emb, sc = torch.from_numpy(table).cuda(), torch.from_numpy(scales).cuda()
    prompt = torch.from_numpy(synth.prompt_ids(T, sh.vocab)).cuda()
    kv = S.KVCache(plan.desc, 1, T + n_new + 80)
    ids = plan.generate(emb, sc, prompt, n_new, kv)
    torch.cuda.synchronize()
    return plan, emb, sc, prompt, kv, ids.cpu().numpy()


def packed(plan, kv, kind, T, copies):
    """The prompt's rows of a prefilled plan cache, packed into a typed cache of `copies` sequences."""
    L, _, H, S_, dh = kv.k.shape
    c = S.SeqCache.empty(L, copies, H, S_, dh, DTYPES[kind])
    for l in range(L):
        k, v = (t[l, :, :, :T].transpose(1, 2).expand(copies, -1, -1, -1) for t in (kv.k, kv.v))
        S.seq_append(c, l, None, k, v)
    c.len.fill_(T)
    plan.seq_bind(c)
    return c


@pytest.mark.parametrize("graph", [False, True])
def test_greedy_steps_give_greedy_text(graph):
    """Drafts right, partly right and wrong, in trees, for three copies of a prompt: the emitted text is the greedy one.
    With a graph the step is captured once and replayed with new tokens and parents."""
    flush(f"case greedy steps graph={graph}")
    sh = Shape(2, 512, 8, 2, 64, 1536, vocab=512)
    T0, n_new, T = 30, 40, 7
    plan, emb, sc, prompt, kv, text = request(sh, T0, n_new)
    kv2 = S.KVCache(plan.desc, 1, kv.k.shape[3])
    logits = torch.empty((sh.vocab,), device="cuda")
    x = (emb[prompt.long()].float() * sc[prompt.long(), None]).contiguous()
    plan.prefill_last(x, T0, kv2, 0, logits)
    cache = packed(plan, kv2, "bf16", T0, 3)
    tokens = torch.zeros((3, T), dtype=torch.int32, device="cuda")
    parent = torch.zeros((3, T), dtype=torch.int32, device="cuda")
    ws = plan.tree_workspace(cache, T)
    scratch = (torch.empty((3, T, sh.d_model), device="cuda"), torch.empty((3, T, sh.vocab), device="cuda"))
    out = (torch.empty((3, T), dtype=torch.int32, device="cuda"), torch.empty((3, T), dtype=torch.int32, device="cuda"),
           torch.empty((3,), dtype=torch.int32, device="cuda"))
    step = lambda: plan.tree_step(emb, sc, tokens, cache, parent=parent, out=out, scratch=scratch, workspace=ws)  # noqa: E731
    g = None
    if graph:
        keep = cache.len.clone()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step()                      # once outside, as a program would
        side.synchronize()
        cache.len.copy_(keep)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        cache.len.copy_(keep)
        torch.cuda.synchronize()
    rng = np.random.default_rng(1)
    done = [1, 1, 1]                    # text[0] follows the prompt: the first node 0
    got = [[int(text[0])] for _ in range(3)]
    for _ in range(60):
        if min(done) > n_new - T:
            break
        tk, pa = np.zeros((3, T), np.int32), np.zeros((3, T), np.int32)
        for b in range(3):
            tk[b, 0], pa[b, 0] = got[b][-1], -1
            depth = [0] * T
            for t in range(1, T):
                pa[b, t] = t - 1 if b == 0 else rng.integers(max(0, t - 3), t)
                depth[t] = depth[pa[b, t]] + 1
                at = done[b] + depth[t] - 1
                right = at < len(text) and (b == 0 or rng.random() < (0.7 if b == 1 else 0.2))
                tk[b, t] = text[at] if right else rng.integers(0, sh.vocab)
            if b == 2:
                pa[b, T - 2:] = -2
        tokens.copy_(torch.from_numpy(tk))
        parent.copy_(torch.from_numpy(pa))
        before, left = cache.len.tolist(), len(text) - done[0]
        g.replay() if graph else step()
        torch.cuda.synchronize()
        ids, path, n = (t.cpu().numpy() for t in out)
        for b in range(3):
            new = ids[b, :n[b]].tolist()
            got[b] += new
            done[b] += len(new)
            assert cache.len[b].item() == before[b] + n[b] == T0 + done[b] - 1
        assert n[0] >= 1 + min(T - 1, max(left, 0))     # sequence 0 drafts the text itself, up to its end
    for b in range(3):
        m = min(len(got[b]), len(text))
        assert m > 20 and got[b][:m] == text[:m].tolist(), b


def test_drafting_with_a_pruned_plan():
    """A sparser plan of the same store drafts a chain greedily on its own cache, the dense plan verifies it by
    sampling from an INT8 cache; steps repeat bit for bit."""
    flush("case draft with a pruned plan")
    sh = Shape(2, 512, 8, 2, 64, 1536, vocab=512)
    T0, T = 20, 5
    store, fn, lm, dense = plan_of(sh, None, 64, 128)
    q = np.ones((2, 8), np.uint8)
    q[:, 1] = 0
    f = np.ones((2, 1536), np.uint8)
    f[:, 1024:] = 0
    sparse = S.Plan(dense.desc, dense.store, (q, None, f))
    table, scales = synth.embedding(sh)
    emb, sc = torch.from_numpy(table).cuda(), torch.from_numpy(scales).cuda()
    prompt = torch.from_numpy(synth.prompt_ids(T0, sh.vocab)).cuda()
    kv = S.KVCache(dense.desc, 1, 128)
    logits = torch.empty((sh.vocab,), device="cuda")
    dense.prefill_last((emb[prompt.long()].float() * sc[prompt.long(), None]).contiguous(), T0, kv, 0, logits)
    runs = []
    for _ in range(2):
        cache = packed(dense, kv, "int8", T0, 1)
        text = [int(logits.argmax())]
        g = gen(9)
        for _ in range(6):
            ctx = torch.cat([prompt, torch.tensor(text, dtype=torch.int32, device="cuda")])
            draft = sparse.generate(emb, sc, ctx, T - 2, S.KVCache(sparse.desc, 1, 128))
            tokens = torch.cat([ctx[-1:], draft])[None].contiguous()
            u = torch.rand((1, T), generator=g).cuda()
            ids, path, n = dense.tree_step(emb, sc, tokens, cache, u=u, temperature=0.8)
            torch.cuda.synchronize()
            assert cache.len.item() == T0 + len(text) - 1 + n.item()
            text += ids[0, :n.item()].tolist()
            assert all(0 <= t < sh.vocab for t in text)
        runs.append(text)
    assert runs[0] == runs[1]


def test_step_refusals():
    flush("case step refusals")
    sh = Shape(1, 512, 8, 2, 64, 1536, vocab=100)
    store, fn, lm, plan = plan_of(sh, None, 16, 64)
    c = S.SeqCache.empty(1, 2, 2, 64, 64, torch.int8)
    x = torch.zeros((2, 4, 512), device="cuda")

    def refused(status, f):
        with pytest.raises(B.TaspError) as e:
            f()
        assert B.STATUS[e.value.status] == status

    refused("TASP_ERR_CACHE_PLAN_MISMATCH", lambda: plan.tree_forward(x, c))
    refused("TASP_ERR_SHAPE", lambda: plan.seq_bind(S.SeqCache.empty(2, 2, 2, 64, 64)))
    refused("TASP_ERR_SHAPE", lambda: plan.seq_bind(S.SeqCache.empty(1, 2, 2, 64, 128)))
    plan.seq_bind(c)
    refused("TASP_ERR_SHAPE", lambda: plan.tree_forward(torch.zeros((2, 9, 512), device="cuda"), c))   # 18 nodes
    ws = plan.tree_workspace(c, 4, 64)
    refused("TASP_ERR_INVALID_ARG", lambda: B.tasp_tree_forward(plan.handle, x.data_ptr(), None, 4, c.struct, 64,
                                                               x.data_ptr(), ws[1], ws[2], None))
    emb, sc = torch.zeros((100, 512), dtype=torch.int8, device="cuda"), torch.zeros(100, device="cuda")
    tk = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    refused("TASP_ERR_INVALID_ARG", lambda: plan.tree_step(emb, sc, tk, c, temperature=1.0))           # no random numbers
    refused("TASP_ERR_WORKSPACE", lambda: plan.tree_step(emb, sc, tk, c, workspace=(None, ws[1], 16)))
    with pytest.raises(ValueError):
        plan.tree_step(emb, sc, tk[:1], c)
    headless = plan_of(Shape(1, 512, 8, 2, 64, 1536), None, 16, 64)[3]
    headless.seq_bind(c)
    refused("TASP_ERR_UNSUPPORTED", lambda: headless.tree_step(emb[:0], sc[:0], tk, c))
    assert c.len.tolist() == [0, 0]


def test_drafts_outside_the_vocabulary():
    """Tokens outside the vocabulary in a branch: they are not accepted, and the other branch goes on as without them."""
    flush("case drafts outside the vocabulary")
    sh = Shape(2, 512, 8, 2, 64, 1536, vocab=512)
    T0 = 30
    plan, emb, sc, prompt, kv, text = request(sh, T0, 8)
    kv2 = S.KVCache(plan.desc, 1, kv.k.shape[3])
    x = (emb[prompt.long()].float() * sc[prompt.long(), None]).contiguous()
    plan.prefill_last(x, T0, kv2, 0, torch.empty((sh.vocab,), device="cuda"))
    parent = torch.tensor([[-1, 0, 0, 2, 3, 1]], dtype=torch.int32, device="cuda")      # 0 - 2 - 3 - 4 and 0 - 1 - 5
    right = [int(t) for t in text[:4]]
    outs = []
    for kind in ("bf16", "int8"):
        for wrong in ((7, 9), (-5, 512), (2 ** 31 - 1, -2 ** 31)):
            cache = packed(plan, kv2, kind, T0, 1)
            tokens = torch.tensor([[right[0], wrong[0], right[1], right[2], right[3], wrong[1]]], dtype=torch.int32, device="cuda")
            ids, path, n = plan.tree_step(emb, sc, tokens, cache, parent=parent)
            torch.cuda.synchronize()
            k, v = S.seq_read(cache, 1, T0 + 6)
            outs.append((ids.tolist(), path.tolist(), cache.len.item(), k[:, :, :T0 + 4].isfinite().all().item() and v[:, :, :T0 + 4].isfinite().all().item()))
            assert path.tolist() == [[0, 2, 3, 4, -1, -1]] and outs[-1][3]
        assert outs[-1] == outs[-2] == outs[-3]
