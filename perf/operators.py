"""Timed calls of the drafted-token operators, each beside its plain form and its definition in 64 bits.

Four operators that together verify drafted tokens against a plan's model:

  append  rotary positions of q and k (half or interleaved pairs, part of the head, scaled for long
          contexts), k and v written into a cache of BF16, INT8 or E4M3 rows (8 bits: one float32
          scale per row and head, the row's largest magnitude over the largest code), and the
          written rows read back as BF16
  attn    attention of T nodes per sequence over its cached rows and, among the nodes' own rows,
          over each node's ancestors and itself (a tree given by parents; none: a chain)
  verify  drafted tokens against the target's probabilities at given random numbers: acceptance
          along the tree, then one token from what is left of the distribution
  commit  the accepted path's cache rows moved together behind the sequence

Node t of a sequence with `len` cached rows has row len + t, position len + its depth, and sees rows
0 .. len - 1, its ancestors' rows and its own. A parent of -1 is a root, anything else outside 0 .. t - 1
an absent node (shorter trees in a batch): zeros as q and as attention output, never accepted, not written.

verify, per sequence: node 0 is the last token already in the text, nodes t >= 1 are drafted tokens x_t
behind their parents, p_v = softmax(logits[v] / temperature). At the current node v its children are
tried in order. Without draft logits child c is accepted when u_c (1 - sum of p_v over the earlier
children's distinct tokens) < p_v(x_c), the mass of a token tried before being 0; with them (chains) when
u_c q_v(x_c) < p_v(x_c), q = softmax(draft logits / temperature). An accepted child becomes the current
node; where none is accepted, the last token is the lowest x whose cumulative weight exceeds u_0 times
the total weight, the weights being p_v without the children's tokens, or max(p_v - q_v, 0). Temperature
0 stands for the distribution on the lowest index of the largest logit.

The 8B and 70B head counts are those of Llama-3 (32 / 8 and 64 / 8 heads of 128), 24 / 3 heads of 64
a generic odd model; vocabulary 128256.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
QMAX = {"int8": 127.0, "e4m3": 448.0}
V3 = 128256


def _append(hq, hkv, dh, batch, T, length, cache, act="bf16", tree=False, layout="half", rot=None,
            scaling="none"):
    return dict(kind="append", hq=hq, hkv=hkv, dh=dh, batch=batch, T=T, len=length, cache=cache, act=act,
                tree=tree, layout=layout, rot=dh if rot is None else rot, scaling=scaling)


def _attn(hq, hkv, dh, batch, T, length, cache, act="bf16", tree=True):
    return dict(kind="attn", hq=hq, hkv=hkv, dh=dh, batch=batch, T=T, len=length, cache=cache, act=act, tree=tree)


def _verify(batch, T, vocab, tree=False, draft=False, temperature=1.0):
    return dict(kind="verify", batch=batch, T=T, vocab=vocab, tree=tree, draft=draft, temperature=temperature)


def _commit(layers, hkv, dh, batch, T, n, max_seq):
    return dict(kind="commit", layers=layers, hkv=hkv, dh=dh, batch=batch, T=T, n=n, max_seq=max_seq)


def listed():
    return [
        # trees of a batch (latency) behind long ragged contexts: interleaved pairs, half of the head, scaled positions
        dict(name="append_tree", **_append(64, 8, 128, 8, 32, 100000, "e4m3", tree=True, layout="interleaved",
                                           rot=64, scaling="wavelength")),
        # a whole prompt's rows into an 8-bit cache and back, float32 activations as the plans have them
        dict(name="append_prompt", **_append(32, 8, 128, 2, 8192, 0, "int8", act="f32")),
        # the next token of one conversation over an 8-bit cache (the form for single tokens)
        dict(name="attn_token", **_attn(32, 8, 128, 1, 1, 2047, "int8", tree=False)),
        # a chunk on an odd model with heads of 64, float32, ragged batch, BF16 cache
        dict(name="attn_odd_f32", **_attn(24, 3, 64, 3, 5, 1001, "bf16", act="f32")),
        # a tree of 16 for four conversations of different lengths, BF16 cache
        dict(name="attn_tree", **_attn(32, 8, 128, 4, 16, 4096, "bf16")),
        # eight drafted tokens behind a context of 128 Ki rows in E4M3
        dict(name="attn_long", **_attn(32, 8, 128, 1, 8, 131064, "e4m3")),
        # the widest tree over eight 70B conversations: the matrix cores' end of the range
        dict(name="attn_wide", **_attn(64, 8, 128, 8, 64, 8192, "int8")),
        # plain sampling of one token
        dict(name="verify_sample", **_verify(1, 1, V3, temperature=0.7)),
        # chains of eight drawn from a draft model's distributions, batch of 8
        dict(name="verify_chain", **_verify(8, 9, V3, draft=True, temperature=0.8)),
        # trees of 32 for 16 conversations (the largest call)
        dict(name="verify_tree", **_verify(16, 32, V3, tree=True)),
        # an accepted path of 5 nodes out of 16 in every layer of an 8B cache
        dict(name="commit_8b", **_commit(32, 8, 128, 1, 16, 5, 1024)),
        # nine of 64 in every layer of eight 70B caches
        dict(name="commit_70b", **_commit(80, 8, 128, 8, 64, 9, 256)),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("append", "attn", "attn", "verify", "commit"))
    hq, hkv, dh = rng.choice(((32, 8, 128), (64, 8, 128), (24, 3, 64), (8, 2, 64), (28, 4, 128), (16, 16, 128), (9, 3, 64)))
    cache = rng.choice(("bf16", "int8", "e4m3"))
    act = rng.choice(("bf16", "bf16", "f32"))
    if kind == "append":
        tree = rng.random() < 0.5
        T = rng.randint(1, 64) if tree else _log(rng, 1, 8192)
        batch = _log(rng, 1, max(1, min(16, 16384 // T)))
        return _append(hq, hkv, dh, batch, T, rng.choice((0, _log(rng, 1, 200000 // batch))) if T <= 64 else 0, cache, act, tree,
                       rng.choice(("half", "interleaved")), rng.choice((dh, dh // 2, dh - 16)),
                       rng.choice(("none", "linear", "wavelength", "index")))
    if kind == "attn":
        T = rng.choice((1, _log(rng, 1, 64), _log(rng, 1, 64)))
        batch = _log(rng, 1, 16)
        most = min(131000.0, 2.4e8 / (batch * hkv * dh * (2 if cache == "bf16" else 1) * 2), 1.2e11 / (4.0 * batch * hq * T * dh))
        return _attn(hq, hkv, dh, batch, T, rng.choice((0, _log(rng, 1, most), _log(rng, 64, most), _log(rng, 64, most))),
                     cache, act, rng.random() < 0.7)
    if kind == "verify":
        vocab = rng.choice((V3, 32000, _log(rng, 2, 150000)))
        draft = rng.random() < 0.4
        T = _log(rng, 1, 64)
        batch = _log(rng, 1, max(1, min(32, int(6e7 / (vocab * T * (2 if draft else 1))))))
        return _verify(batch, T, vocab, not draft and rng.random() < 0.7, draft, rng.choice((0.0, 0.3, 0.7, 1.0, 1.3)))
    T = _log(rng, 1, 64)
    return _commit(_log(rng, 1, 80), hkv, dh, _log(rng, 1, 8), T, rng.randint(1, T), rng.choice((96, 130, 256)))


# ----------------------------------------------------------------------------------- inputs

def _lens(case):
    """Cached rows of each sequence: the first has `len`, the others down to about half of it."""
    return [case["len"] - b * case["len"] // (2 * case["batch"]) for b in range(case["batch"])]


def _parents(case, gen):
    """Random trees: a node hangs off one of the eight before it; every third sequence misses its last nodes."""
    B, T = case["batch"], case["T"]
    t = torch.arange(T)
    back = 1 + (torch.rand((B, T), generator=gen) * torch.clamp(t, 1, 8)).long()
    p = torch.clamp(t - torch.minimum(back, torch.clamp(t, min=1)), min=-1)
    p[:, 0] = -1
    count = torch.tensor([max(1, T - T // 4) if b % 3 == 2 else T for b in range(B)])
    return torch.where(t < count[:, None], p, torch.tensor(-2)).to(torch.int32)


def _rope(case):
    d = dict(theta=500000.0, factor=1.0, low=1.0, high=4.0, orig_len=8192, mscale=1.0)
    if case["scaling"] == "linear":
        d.update(factor=4.0)
    if case["scaling"] == "wavelength":
        d.update(factor=8.0)
    if case["scaling"] == "index":
        d.update(factor=16.0, low=1.0, high=32.0, mscale=0.1 * math.log(16.0) + 1.0)
    return d


def _randn(gen, shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device=DEV).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    host = torch.Generator().manual_seed(int(seed))
    B, T = case["batch"], case["T"]
    s = {"case": case}
    if case["kind"] in ("append", "attn"):
        H, dh, dt = case["hkv"], case["dh"], TYPES[case["cache"]]
        rows = case["len"] + T + 3
        rows = (rows + 15) // 16 * 16
        act = TYPES[case["act"]]
        s["len"] = torch.tensor(_lens(case), dtype=torch.int32, device=DEV)
        s["parent"] = _parents(case, host).to(DEV) if case["tree"] else None
        s["q"] = _randn(gen, (B, T, case["hq"], dh), act)
        if case["kind"] == "append":
            # one fused projection's output: q, k and v of a token side by side
            qkv = torch.cat([s["q"].flatten(2), _randn(gen, (B, T, 2 * H * dh), act)], -1)
            n = case["hq"] * dh
            s["q"] = qkv[..., :n].unflatten(-1, (case["hq"], dh))
            s["k"] = qkv[..., n:n + H * dh].unflatten(-1, (H, dh))
            s["v"] = qkv[..., n + H * dh:].unflatten(-1, (H, dh))
            s["rope"] = _rope(case)
        shape = (1, B, H, rows, dh)
        for name in ("kc", "vc"):
            if case["kind"] == "append":
                s[name] = torch.zeros(shape, dtype=dt, device=DEV)
                s[name + "_scale"] = torch.zeros(shape[:-1], device=DEV) if case["cache"] in QMAX else None
                continue
            x = _randn(gen, shape)
            if name == "kc":           # a few large channels, as keys have them
                x[..., :: 16] *= 3.0
            if case["cache"] in QMAX:
                sc = x.abs().amax(-1) / QMAX[case["cache"]]
                x = x / sc[..., None]
                s[name] = (x.round() if case["cache"] == "int8" else x).clamp(-QMAX[case["cache"]], QMAX[case["cache"]]).to(dt)
                s[name + "_scale"] = sc
            else:
                s[name], s[name + "_scale"] = x.to(dt), None
    elif case["kind"] == "verify":
        V = case["vocab"]
        s["parent"] = _parents(case, host).to(DEV) if case["tree"] else None
        s["u"] = torch.rand((B, T), generator=gen, device=DEV)
        base = _randn(gen, (B, T, V)) * 2.5
        if case["temperature"] == 0:       # ties of the largest logit occur
            base = base.to(torch.bfloat16).float()
        s["logits"] = base
        s["draft"] = base[:, :T - 1] + _randn(gen, (B, T - 1, V)) * 0.7 if case["draft"] else None
        # a drafted token is drawn from the draft's distribution, or is one of the target's likely ones
        tokens = torch.zeros((B, T), dtype=torch.int32, device=DEV)
        if T > 1:
            from_ = s["draft"] if case["draft"] else base
            up = s["parent"].long().clamp(min=0)[:, 1:, None] if case["tree"] else torch.arange(T - 1, device=DEV).expand(B, -1)[..., None]
            row = torch.gather(from_, 1, up.expand(-1, -1, V)) / max(case["temperature"], 0.5)
            tokens[:, 1:] = (row - torch.empty_like(row).exponential_(generator=gen).log()).argmax(-1).to(torch.int32)
            if not case["draft"]:          # most drafts are good ones
                best = row.argmax(-1).to(torch.int32)
                tokens[:, 1:] = torch.where(torch.rand((B, T - 1), generator=gen, device=DEV) < 0.4, best, tokens[:, 1:])
        s["tokens"] = tokens
    else:
        shape = (case["layers"], B, case["hkv"], case["max_seq"], case["dh"])
        s["kc"], s["vc"] = _randn(gen, shape, torch.bfloat16), _randn(gen, shape, torch.bfloat16)
        n, far = case["n"], case["T"] - case["n"]
        steps = torch.sort(torch.rand((B, max(0, n - 1)), generator=host) * far, dim=1).values.ceil().long()
        path = torch.full((B, T), -1, dtype=torch.int32)
        path[:, 0] = 0
        path[:, 1:n] = (torch.arange(1, n) + steps).to(torch.int32)
        s["path"] = path.to(DEV)
        s["n"] = torch.full((B,), n, dtype=torch.int32, device=DEV)
        s["len"] = torch.tensor([(case["max_seq"] - T) // (b + 1) for b in range(B)], dtype=torch.int32, device=DEV)
    return s


# ----------------------------------------------------------------------------------- one pass

def run(s):
    if own:
        return _own(s)
    return {"append": _append_plain, "attn": _attn_plain, "verify": _verify_plain, "commit": _commit_plain}[s["case"]["kind"]](s)


def _own(s):
    from paper_2609_29499_amd import session as S

    c = s["case"]
    if c["kind"] == "verify":
        if "ws" not in s:
            s["ws"] = S.verify_workspace(c["batch"], c["T"], c["vocab"], DEV)
        ids, path, n = S.verify(s["logits"], s["tokens"], s["u"], s["parent"], s["draft"], c["temperature"], workspace=s["ws"])
        return {"ids": ids, "path": path, "n": n}
    if "cache" not in s:
        s["cache"] = S.SeqCache(s["kc"], s["vc"], s["len"], s.get("kc_scale"), s.get("vc_scale"))
        if c["kind"] == "append":
            s["rotary"] = S.Rope(c["layout"], c["rot"], scaling=c["scaling"], **s["rope"])
        if c["kind"] == "attn":
            s["ws"] = S.tree_attention_workspace(s["cache"], c["hq"], c["T"], c["len"])
    if c["kind"] == "append":
        q = S.seq_append(s["cache"], 0, s["q"], s["k"], s["v"], s["rotary"], s["parent"])
        k, v = S.seq_read(s["cache"], 0, c["T"], first=s["len"])
        return {"q": q, "k": k, "v": v}
    if c["kind"] == "attn":
        return S.tree_attention(s["cache"], 0, s["q"], s["parent"], max_len=c["len"], workspace=s["ws"])
    now = S.seq_commit(s["cache"], s["path"], s["n"], len_out=torch.empty_like(s["len"]))
    return {"k": s["kc"], "v": s["vc"], "len": now}


def _tree(s):
    """present [B, T], seen [B, T, T] (column j is an ancestor of node t or t itself), depth [B, T]."""
    B, T = s["case"]["batch"], s["case"]["T"]
    t = torch.arange(T, device=DEV)
    if s["parent"] is None:
        return torch.ones((B, T), dtype=torch.bool, device=DEV), (t <= t[:, None]).expand(B, T, T), t.expand(B, T)
    up = (s["parent"][..., None] == t).double() + torch.eye(T, dtype=torch.float64, device=DEV)
    seen = torch.linalg.matrix_power(up, 64) > 0       # every chain of parents is shorter than 64
    return s["parent"] >= -1, seen, seen.sum(-1) - 1


def _frequencies(c, d, device):
    i = torch.arange(0, c["rot"], 2, dtype=torch.float64, device=device)
    inv = torch.exp(-math.log(d["theta"]) * i / c["rot"])
    if c["scaling"] == "linear":
        return inv / d["factor"]
    if c["scaling"] == "wavelength":       # by the turns that a pair makes over the original length
        keep = ((d["orig_len"] * inv / (2 * math.pi) - d["low"]) / (d["high"] - d["low"])).clamp(0, 1)
        return inv * (keep + (1 - keep) / d["factor"])
    if c["scaling"] == "index":            # by the pair's index, between the pairs that make `high` and `low` turns
        at = [c["rot"] * math.log(d["orig_len"] / (2 * math.pi * x)) / (2 * math.log(d["theta"])) for x in (d["high"], d["low"])]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), c["rot"] - 1)
        ramp = ((i / 2 - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return inv * ((1 - ramp) + ramp / d["factor"])
    return inv


def _rotate(c, x, cos, sin):
    n = c["rot"]
    if c["layout"] == "half":
        a, b = x[..., :n // 2], x[..., n // 2:n]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., n:]], -1)
    a, b = x[..., 0:n:2], x[..., 1:n:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., n:]], -1)


def _bits(x):
    """E4M3 as plain bytes, for indexing."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _store(s, name, x, where):
    """x [B, T, H, dh] float32 into the cache rows `where` ([B, T], -1: nowhere)."""
    c = s["case"]
    if c["cache"] in QMAX:
        # in 64 bits and by division: x qmax / top may lie on the border between two codes
        top = x.abs().amax(-1, keepdim=True).double()
        x = (x.double() * QMAX[c["cache"]] / torch.where(top > 0, top, 1.0)).float()
        sc = (top / torch.full_like(top, QMAX[c["cache"]]))[..., 0].float()
        x = (x.round() if c["cache"] == "int8" else x).clamp(-QMAX[c["cache"]], QMAX[c["cache"]])
    b, t = torch.nonzero(where >= 0, as_tuple=True)
    _bits(s[name])[0].transpose(1, 2)[b, where[b, t]] = _bits(x[b, t].to(TYPES[c["cache"]]))
    if c["cache"] in QMAX:
        s[name + "_scale"][0].transpose(1, 2)[b, where[b, t]] = sc[b, t]


def _values(x, scale):
    return x.float() if scale is None else x.float() * scale[..., None]


def _read(s, name, rows):
    """The cache's rows `rows` [B, T] as BF16 [B, H, T, dh]."""
    c = s["case"]
    at = rows[:, None, :].expand(-1, c["hkv"], -1)
    x = torch.gather(_bits(s[name])[0], 2, at[..., None].expand(-1, -1, -1, c["dh"])).view(TYPES[c["cache"]])
    scale = s[name + "_scale"]
    return _values(x, None if scale is None else torch.gather(scale[0], 2, at)).to(torch.bfloat16)


def _append_plain(s):
    c, d = s["case"], s["rope"]
    t = torch.arange(c["T"], device=DEV).expand(c["batch"], -1)
    present, depth = torch.ones_like(t, dtype=torch.bool), t
    if c["tree"]:
        present, _, depth = _tree(s)
    angle = (s["len"].double()[:, None] + depth)[..., None] * _frequencies(c, d, DEV)
    cos, sin = ((f(angle) * d["mscale"]).float()[:, :, None] for f in (torch.cos, torch.sin))
    rows = s["len"].long()[:, None] + t
    where = torch.where(present, rows, -1)
    _store(s, "kc", _rotate(c, s["k"].float(), cos, sin), where)
    _store(s, "vc", s["v"].float(), where)
    q = torch.where(present[..., None, None], _rotate(c, s["q"].float(), cos, sin), 0.0)
    return {"q": q.to(TYPES[c["act"]]), "k": _read(s, "kc", rows), "v": _read(s, "vc", rows)}


def _attn_plain(s):
    c = s["case"]
    B, T, H, dh = c["batch"], c["T"], c["hkv"], c["dh"]
    G, R = c["hq"] // H, s["kc"].shape[3]
    present, seen, _ = _tree(s)
    row = torch.arange(R, device=DEV)
    node = row[None] - s["len"].long()[:, None]        # [B, R]
    new = torch.gather(seen, 2, node.clamp(0, T - 1)[:, None].expand(B, T, R)) & ((node >= 0) & (node < T))[:, None]
    vis = ((node < 0)[:, None] | new) & present[..., None]
    q = s["q"].float().reshape(B, T, H, G, dh).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, dh)
    score = torch.matmul(q, _values(s["kc"][0], None if s["kc_scale"] is None else s["kc_scale"][0]).transpose(2, 3).contiguous()) / math.sqrt(dh)
    score = score.reshape(B, H, T, G, R).masked_fill(~vis[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    v = _values(s["vc"][0], None if s["vc_scale"] is None else s["vc_scale"][0])
    o = torch.matmul(p.reshape(B, H, T * G, R), v).reshape(B, H, T, G, dh)
    o = torch.where(total > 0, o / total, 0.0)
    return o.permute(0, 2, 1, 3, 4).reshape(B, T, c["hq"], dh).to(TYPES[c["act"]])


def _verify_plain(s):
    c = s["case"]
    B, T, V = c["batch"], c["T"], c["vocab"]
    greedy = c["temperature"] == 0
    ids = torch.arange(V, device=DEV)
    t = torch.arange(T, device=DEV)
    x = s["logits"]
    top = x.amax(-1, keepdim=True)
    first = torch.where(x == top, ids, V).amin(-1)                                # [B, T]
    if greedy:
        weight = (ids == first[..., None]).double()
    else:
        weight = torch.exp((x.double() - top.double()) / c["temperature"])
    present, seen, depth = _tree(s)
    up = torch.cat([torch.full((1,), -1, device=DEV), t[:-1]]).expand(B, T) if s["parent"] is None else s["parent"].long()
    total = weight.sum(-1)
    pv = up.clamp(min=0)
    token = s["tokens"].long()
    mine = weight[torch.arange(B, device=DEV)[:, None], pv, token]                # weight of a node's token at its parent
    u = s["u"].double()
    if c["draft"] and not greedy:
        y = s["draft"]
        ew = torch.exp((y.double() - y.amax(-1, keepdim=True).double()) / c["temperature"])
        q = ew / ew.sum(-1, keepdim=True)                                         # [B, T - 1, V]
        qt = torch.cat([torch.ones((B, 1), dtype=torch.float64, device=DEV), torch.gather(q, 2, token[:, 1:, None])[..., 0]], 1)
        good = u * qt < mine / torch.gather(total, 1, pv)
    else:
        older = (up[:, :, None] == up[:, None, :]) & (t < t[:, None]) & present[:, None, :]     # earlier siblings
        same = older & (token[:, :, None] == token[:, None, :])
        fresh = torch.where(same.any(-1), 0.0, mine)
        left = torch.gather(total, 1, pv) - torch.where(older, fresh[:, None, :], 0.0).sum(-1)
        good = u * left < fresh
    good = good & present & (up >= 0)
    older = (up[:, :, None] == up[:, None, :]) & (t < t[:, None])
    good = good & ~(older & good[:, None, :]).any(-1)                             # the first accepted child
    good[:, 0] = True
    on = present & (~seen | good[:, None, :]).all(-1) & seen[..., 0]              # every node up to the root accepted
    last = torch.where(on, depth * T + t, -1).argmax(-1)                          # one node of each depth is on the path
    n = on.sum(-1)
    b = torch.arange(B, device=DEV)
    w = weight[b, last]
    child = present & (up == last[:, None])                                       # [B, T]
    if c["draft"] and not greedy and T > 1:
        p = w / total[b, last][:, None]
        rest = torch.where(child.any(-1)[:, None], (p - q[b, last.clamp(max=T - 2)]).clamp(min=0), p)
    else:
        p = w
        gone = torch.zeros((B, V), device=DEV).scatter_add_(1, token, child.float()) > 0
        rest = torch.where(gone, 0.0, w)
    rest = torch.where(rest.sum(-1, keepdim=True) > 0, rest, p)
    cum = rest.cumsum(-1)
    hit = cum > u[:, :1] * cum[:, -1:]
    new = torch.where(hit, ids, V).amin(-1)
    new = torch.where(new < V, new, torch.where(rest > 0, ids, -1).amax(-1))
    # path: the nodes by depth; ids: the accepted tokens and the new one
    slot = torch.where(on, depth, T)
    path = torch.full((B, T + 1), -1, device=DEV).scatter_(1, slot, t.expand(B, T))[:, :T]
    out = torch.full((B, T + 1), -1, device=DEV).scatter_(1, torch.where(on & (t > 0), depth - 1, T), token)[:, :T]
    out = torch.where(t == (n - 1)[:, None], new[:, None], torch.where(t < (n - 1)[:, None], out, -1))
    return {"ids": out.to(torch.int32), "path": path.to(torch.int32), "n": n.to(torch.int32)}


def _commit_plain(s):
    c = s["case"]
    B, T = c["batch"], c["T"]
    i = torch.arange(T, device=DEV)
    b = torch.arange(B, device=DEV)[:, None]
    src = s["len"].long()[:, None] + torch.where(i < s["n"][:, None], s["path"].long(), i)
    dst = s["len"].long()[:, None] + i
    s["kc"][:, b, :, dst] = s["kc"][:, b, :, src]
    s["vc"][:, b, :, dst] = s["vc"][:, b, :, src]
    return {"k": s["kc"], "v": s["vc"], "len": s["len"] + s["n"]}


# ----------------------------------------------------------------------------------- what a pass costs

def work(case):
    B, T = case["batch"], case["T"]
    size = {"bf16": 2, "f32": 4, "int8": 1, "e4m3": 1}
    if case["kind"] == "verify":
        rows = B * T + (B * (T - 1) if case["draft"] else 0)
        return {"bytes": rows * case["vocab"] * 4.0, "flops": rows * case["vocab"] * 4.0}
    if case["kind"] == "commit":
        moved = 2.0 * case["layers"] * B * case["hkv"] * (case["n"] - 1) * case["dh"] * 2
        return {"bytes": 2 * moved + 8.0 * B * T, "flops": 0.0}
    row = case["dh"] * size[case["cache"]] + (4 if case["cache"] in QMAX else 0)
    if case["kind"] == "append":
        tokens = B * T
        acts = (2 * case["hq"] + 2 * case["hkv"]) * case["dh"] * size[case["act"]]
        kv = 2 * case["hkv"] * (2 * row + 2 * case["dh"])
        return {"bytes": float(tokens * (acts + kv)), "flops": tokens * (case["hq"] + 2.0 * case["hkv"]) * case["dh"] * 3}
    rows = sum(_lens(case)) + B * T
    acts = 2 * B * T * case["hq"] * case["dh"] * size[case["act"]]
    return {"bytes": float(rows * case["hkv"] * 2 * row + acts), "flops": 4.0 * rows * T * case["hq"] * case["dh"]}


# ----------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    if case["kind"] in ("verify", "commit"):
        return None                                    # whole numbers and moved rows
    s = prepare(case, seed)
    B, T, H, dh = case["batch"], case["T"], case["hkv"], case["dh"]
    lens = s["len"].tolist()
    parent = s["parent"].tolist() if s["parent"] is not None else [list(range(-1, T - 1))] * B
    line = []                                          # per sequence and node: itself and its ancestors, or None
    for b in range(B):
        line.append([])
        for t in range(T):
            p = parent[b][t]
            above = [] if p == -1 else line[b][p] if 0 <= p < t else None
            line[b].append(None if above is None else above + [t] if T <= 64 else range(t + 1))
    return _exact_attn(case, s, lens, line) if case["kind"] == "attn" else _exact_append(case, s, lens, line)


def _exact_attn(case, s, lens, line):
    B, T, H, dh = case["batch"], case["T"], case["hkv"], case["dh"]
    G = case["hq"] // H
    out = torch.zeros((B, T, case["hq"], dh), dtype=torch.float64, device=DEV)
    for b in range(B):
        L = lens[b]
        kd, vd = (s[n][0, b, :, :L + T].to(torch.float64) for n in ("kc", "vc"))
        if case["cache"] in QMAX:
            kd = kd * s["kc_scale"][0, b, :, :L + T, None].double()
            vd = vd * s["vc_scale"][0, b, :, :L + T, None].double()
        hide = torch.zeros((T, L + T), dtype=torch.float64, device=DEV)
        hide[:, L:] = -math.inf
        nodes = [t for t in range(T) if line[b][t] is not None]
        for t in nodes:
            hide[t, torch.tensor([L + j for j in line[b][t]], device=DEV)] = 0.0
        for h in range(H):
            x = s["q"][b, :, h * G:(h + 1) * G].double()                          # [T, G, dh]
            z = (x.reshape(-1, dh) @ kd[h].T).reshape(T, G, -1) * dh ** -0.5 + hide[:, None]
            a = torch.exp(z[nodes] - torch.logsumexp(z[nodes], -1, keepdim=True))
            o = (a.reshape(-1, L + T) @ vd[h]).reshape(len(nodes), G, dh)
            out[b, nodes, h * G:(h + 1) * G] = o
    return out


def _exact_append(case, s, lens, line):
    B, T, H, dh, n = case["batch"], case["T"], case["hkv"], case["dh"], case["rot"]
    d = s["rope"]
    freq = []
    for i in range(n // 2):
        f = d["theta"] ** (-2.0 * i / n)
        turns = d["orig_len"] * f / (2 * math.pi)
        if case["scaling"] == "linear":
            f /= d["factor"]
        elif case["scaling"] == "wavelength":
            f *= 1.0 if turns >= d["high"] else 1 / d["factor"] if turns <= d["low"] else \
                (turns - d["low"]) / (d["high"] - d["low"]) * (1 - 1 / d["factor"]) + 1 / d["factor"]
        elif case["scaling"] == "index":
            lo = max(0, math.floor(n / 2 * math.log(d["orig_len"] / d["high"] / 2 / math.pi) / math.log(d["theta"])))
            hi = min(n - 1, math.ceil(n / 2 * math.log(d["orig_len"] / d["low"] / 2 / math.pi) / math.log(d["theta"])))
            g = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f = f * (1 - g) + f / d["factor"] * g
        freq.append(f)
    pos = torch.tensor([[lens[b] + (len(x) - 1 if x is not None else 0) for x in line[b]] for b in range(B)], dtype=torch.float64, device=DEV)
    there = torch.tensor([[x is not None for x in line[b]] for b in range(B)], device=DEV)
    turn = torch.polar(torch.full((), d["mscale"], dtype=torch.float64, device=DEV), pos[..., None] * torch.tensor(freq, dtype=torch.float64, device=DEV))

    def turned(x):
        x = x.double().clone()
        first, second = (slice(0, n // 2), slice(n // 2, n)) if case["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
        z = torch.complex(x[..., first], x[..., second]) * turn[:, :, None]
        x[..., first], x[..., second] = z.real, z.imag
        return x

    def held(x):
        x = x.transpose(1, 2) * there[:, None, :, None]
        if case["cache"] == "bf16":
            return x
        m = x.abs().amax(-1, keepdim=True)
        m[m == 0] = 1.0
        x = x * QMAX[case["cache"]] / m
        x = torch.round(x) if case["cache"] == "int8" else x.float().to(torch.float8_e4m3fn).double()
        return x * (m / QMAX[case["cache"]])

    return {"q": turned(s["q"]) * there[..., None, None], "k": held(turned(s["k"])), "v": held(s["v"].double())}
