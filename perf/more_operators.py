"""Timed calls of the paged-cache operators and of the scores of tokens, each beside its plain form and its definition in 64 bits.

Three operators that serve many conversations of different lengths in one step of a plan's model:

  append  rotary positions of q and k (half or interleaved pairs, part of the head, scaled for long contexts), k and v
          written into the pages of their sequences, and the rows of the touched pages read back as BF16. Pages hold
          page_rows rows of a KV head in BF16, INT8 or E4M3; 8 bits come with one float32 scale per page and head
  attn    causal attention of the new tokens over their sequences' pages: single tokens, chunks of a prompt behind
          cached rows, whole prompts, and mixtures of them
  score   of every row of logits the log probability, entropy, rank and top alternatives of a given token, and the mean
          log probability of every sequence (what the router takes as a prompt's proxy log probability)

The tokens of a step lie packed: those of sequence b are rows start[b] .. start[b + 1] - 1 of q, k, v (start None: one token
per sequence). Sequence b holds len[b] rows, row r of it in page table[b][r // page_rows] at r % page_rows; its i-th new
token is row and position len[b] + i and sees rows 0 .. len[b] + i.

The scale of a page and head is the largest |value| over 127 or 448 of what was written into it since its row 0 was: a call
that raises it rounds the page's older codes again, code' = round(code old / new); new rows are round(x / scale), all to even.

The 8B and 70B head counts are those of Llama-3 (32 / 8 and 64 / 8 heads of 128), 24 / 3 heads of 64 a generic odd model;
vocabulary 128256.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
QMAX = {"int8": 127.0, "e4m3": 448.0}
V3 = 128256


def _append(hq, hkv, dh, batch, T, length, cache, page, act="bf16", mode="ragged", layout="half", rot=None, scaling="none"):
    return dict(kind="append", hq=hq, hkv=hkv, dh=dh, batch=batch, T=T, len=length, cache=cache, page=page, act=act, mode=mode,
                layout=layout, rot=dh if rot is None else rot, scaling=scaling)


def _attn(hq, hkv, dh, batch, T, length, cache, page, act="bf16", mode="ragged", shared=0):
    return dict(kind="attn", hq=hq, hkv=hkv, dh=dh, batch=batch, T=T, len=length, cache=cache, page=page, act=act, mode=mode,
                shared=shared)


def _score(rows, vocab, top, seqs=1, logits="f32", temperature=1.0):
    return dict(kind="score", rows=rows, vocab=vocab, top=top, seqs=seqs, logits=logits, temperature=temperature)


def listed():
    return [
        # the next token of 64 conversations into half-filled pages, interleaved pairs of half the head, scaled positions
        dict(name="append_step", **_append(32, 8, 128, 64, 1, 30000, "e4m3", 16, mode="one", layout="interleaved", rot=64,
                                           scaling="wavelength")),
        # prompts of a batch into INT8 pages, float32 activations as the plans have them
        dict(name="append_prompts", **_append(64, 8, 128, 4, 3000, 0, "int8", 64, act="f32")),
        # the next token of one conversation (latency, the form for single tokens)
        dict(name="attn_token", **_attn(32, 8, 128, 1, 1, 2047, "int8", 16, mode="one")),
        # one step of 32 conversations that share a system prompt of 1024 rows
        dict(name="attn_step", **_attn(32, 8, 128, 32, 1, 8190, "int8", 64, mode="one", shared=16)),
        # four long conversations of a 70B model in E4M3, one token each
        dict(name="attn_long", **_attn(64, 8, 128, 4, 1, 65530, "e4m3", 128, mode="one")),
        # a few tokens on an odd model with heads of 64, float32, ragged batch, BF16 pages
        dict(name="attn_odd_f32", **_attn(24, 3, 64, 3, 37, 1001, "bf16", 32, act="f32")),
        # a chunk of a prompt of 512 tokens behind 8 Ki rows, in one step with three other conversations' single tokens
        dict(name="attn_chunk", **_attn(32, 8, 128, 4, 512, 8191, "int8", 32, mode="mixed")),
        # a whole prompt of 8 Ki tokens of a 70B model, BF16 pages: the matrix cores' end of the range
        dict(name="attn_prompt", **_attn(64, 8, 128, 1, 8192, 0, "bf16", 64)),
        # the sampled token's log probability with 20 alternatives
        dict(name="score_token", **_score(1, V3, 20)),
        # one step of 64 conversations
        dict(name="score_step", **_score(64, V3, 5, temperature=0.7)),
        # logits in BF16 of an odd vocabulary
        dict(name="score_bf16", **_score(513, 32003, 32, seqs=3, logits="bf16")),
        # prompts scored for the router's proxy log probability: the largest call
        dict(name="score_prompts", **_score(2048, V3, 1, seqs=5)),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("append", "attn", "attn", "score"))
    hq, hkv, dh = rng.choice(((32, 8, 128), (64, 8, 128), (24, 3, 64), (8, 2, 64), (28, 4, 128), (16, 16, 128), (9, 3, 64)))
    cache = rng.choice(("bf16", "int8", "e4m3"))
    act = rng.choice(("bf16", "bf16", "f32"))
    page = rng.choice((16, 32, 64, 128))
    mode = rng.choice(("one", "ragged", "mixed"))
    if kind == "append":
        batch = _log(rng, 1, 128)
        T = 1 if mode == "one" else _log(rng, 1, 12000 // (batch if mode == "ragged" else 1))
        return _append(hq, hkv, dh, batch, T, rng.choice((0, _log(rng, 1, 200000 // batch))), cache, page, act, mode,
                       rng.choice(("half", "interleaved")), rng.choice((dh, dh // 2, dh - 16)),
                       rng.choice(("none", "linear", "wavelength", "index")))
    if kind == "attn":
        batch = _log(rng, 1, 64)
        room = 4.3e9 / (batch * hq)                    # of the plain form's padded scores
        T = 1 if mode == "one" else _log(rng, 1, min(8192.0, math.sqrt(room), 16384 / batch))
        most = min(131000.0, 5e8 / (batch * hkv * dh * (2 if cache == "bf16" else 1)), room / T - T, 1e12 / (4.0 * batch * hq * T * dh))
        length = rng.choice((0, _log(rng, 1, max(1.0, most)), _log(rng, 64, max(64.0, most)), _log(rng, 64, max(64.0, most))))
        return _attn(hq, hkv, dh, batch, T, length, cache, page, act, mode, rng.choice((0, 0, length // (4 * page))))
    vocab = rng.choice((V3, 32003, _log(rng, 2, 150000)))
    rows = _log(rng, 1, min(4096.0, 2.6e8 / vocab))
    return _score(rows, vocab, rng.choice((0, 1, rng.randint(1, 32))), rng.randint(1, min(rows, 8)), rng.choice(("f32", "f32", "bf16")),
                  rng.choice((1.0, 1.0, 0.6, 1.3)))


# ----------------------------------------------------------------------------------- inputs

def _lens(case):
    """Cached rows of each sequence: the first has `len`, the others down to about half of it."""
    return [case["len"] - b * case["len"] // (2 * case["batch"]) for b in range(case["batch"])]


def _counts(case):
    """New tokens of each sequence: one, T down to about half of it, or T of the first and one of the others."""
    if case["mode"] == "ragged":
        return [case["T"] - b * case["T"] // (2 * case["batch"]) for b in range(case["batch"])]
    return [case["T"] if b == 0 else 1 for b in range(case["batch"])]


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
    s = {"case": case}
    if case["kind"] == "score":
        R, V = case["rows"], case["vocab"]
        x = _randn(gen, (R, V)) * 2.5
        s["logits"] = x.to(TYPES[case["logits"]])
        # most tokens are likely ones; a few rows of a batch are padding
        likely = (x + _randn(gen, (R, V)) * 2.0).argmax(-1)
        any_ = torch.randint(0, V, (R,), generator=gen, device=DEV)
        tokens = torch.where(torch.rand((R,), generator=gen, device=DEV) < 0.8, likely, any_).to(torch.int32)
        if R > 16:
            tokens[torch.rand((R,), generator=gen, device=DEV) < 0.02] = -1
        s["tokens"] = tokens
        cut = torch.sort(torch.randperm(R - 1, generator=host)[:case["seqs"] - 1] + 1).values.tolist() if R > 1 else []
        s["start"] = torch.tensor([0] + cut + [R], dtype=torch.int32, device=DEV)
        return s
    B, P, H, dh = case["batch"], case["page"], case["hkv"], case["dh"]
    lens, counts = _lens(case), _counts(case)
    N = sum(counts)
    need = [(n + c + P - 1) // P for n, c in zip(lens, counts)]
    shared = min(case.get("shared", 0), min(n // P for n in lens))
    width = max(need)
    n_pages = sum(need) - shared * (B - 1) + 3
    order = torch.randperm(n_pages, generator=host).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = shared
    for b in range(B):
        table[b, :shared] = order[:shared]
        table[b, shared:need[b]] = order[at:at + need[b] - shared]
        at += need[b] - shared
    s["table"] = table.to(DEV)
    s["len"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["start"] = None
    if case["mode"] != "one":
        s["start"] = torch.tensor([sum(counts[:b]) for b in range(B + 1)], dtype=torch.int32, device=DEV)
    dt, act = TYPES[case["cache"]], TYPES[case["act"]]
    shape = (1, n_pages, H, P, dh)
    for name in ("kc", "vc"):
        x = _randn(gen, shape)
        if name == "kc":               # a few large channels, as keys have them
            x[..., ::16] *= 3.0
        if case["cache"] in QMAX:
            sc = x.abs().amax((-2, -1)) / QMAX[case["cache"]]
            x /= sc[..., None, None]
            s[name] = (x.round_() if case["cache"] == "int8" else x).clamp_(-QMAX[case["cache"]], QMAX[case["cache"]]).to(dt)
            s[name + "_scale"] = sc
        else:
            s[name], s[name + "_scale"] = x.to(dt), None
        del x
    if case["kind"] == "attn":
        s["q"] = _randn(gen, (N, case["hq"], dh), act)
        return s
    # one fused projection's output: q, k and v of a token side by side
    qkv = _randn(gen, (N, (case["hq"] + 2 * H) * dh), act)
    n = case["hq"] * dh
    s["q"] = qkv[:, :n].unflatten(-1, (case["hq"], dh))
    s["k"] = qkv[:, n:n + H * dh].unflatten(-1, (H, dh))
    s["v"] = qkv[:, n + H * dh:].unflatten(-1, (H, dh))
    s["k"][..., ::16] *= 3.0
    s["rope"] = _rope(case)
    s["first"] = s["len"] // P * P     # rows are read back from the start of the page that a sequence continues
    return s


def _read_rows(case):
    return case["T"] + case["page"]


# ----------------------------------------------------------------------------------- one pass

def run(s):
    if own:
        return _own(s)
    return {"append": _append_plain, "attn": _attn_plain, "score": _score_plain}[s["case"]["kind"]](s)


def _own(s):
    from paper_2609_29499_amd import session as S

    c = s["case"]
    if c["kind"] == "score":
        if "ws" not in s:
            s["ws"] = S.token_logprobs_workspace(c["rows"], c["vocab"], c["top"], DEV)
        return S.token_logprobs(s["logits"], s["tokens"], n_top=c["top"], temperature=c["temperature"], start=s["start"],
                                workspace=s["ws"])._asdict()
    if "cache" not in s:
        s["cache"] = S.PageCache(s["kc"], s["vc"], s["table"], s["len"], s["kc_scale"], s["vc_scale"])
        if c["kind"] == "append":
            s["rotary"] = S.Rope(c["layout"], c["rot"], scaling=c["scaling"], **s["rope"])
        else:
            s["ws"] = S.page_attention_workspace(s["cache"], c["hq"], s["q"].shape[0], c["len"], c["T"])
    if c["kind"] == "append":
        q = S.page_append(s["cache"], 0, s["q"], s["k"], s["v"], s["start"], s["rotary"])
        k, v = S.page_read(s["cache"], 0, _read_rows(c), first=s["first"])
        return {"q": q, "k": k, "v": v}
    return S.page_attention(s["cache"], 0, s["q"], s["start"], max_len=c["len"], max_new=c["T"], workspace=s["ws"])


def _tokens(s):
    """Of every token: its sequence and its place among the sequence's new ones; new tokens and first token of every sequence."""
    c, N = s["case"], s["q"].shape[0]
    t = torch.arange(N, device=DEV)
    if s["start"] is None:
        return t, torch.zeros_like(t), torch.ones_like(t), t
    start = s["start"].long()
    b = (t[:, None] >= start[1:]).sum(-1)
    return b, t - start[b], start[1:] - start[:-1], start[:-1]


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


def _codes(c, x):
    """64-bit values in units of the scale as codes."""
    x = x.float()
    return (x.round() if c["cache"] == "int8" else x).clamp(-QMAX[c["cache"]], QMAX[c["cache"]]).to(TYPES[c["cache"]])


def _store(s, name, x):
    """x [N, H, dh] float32 into the pages of their sequences."""
    c = s["case"]
    B, P = c["batch"], c["page"]
    _, _, n, begin = _tokens(s)
    L = s["len"].long()
    J = (c["T"] + P - 2) // P + 1                       # pages that a sequence touches at most
    pg = L[:, None] // P + torch.arange(J, device=DEV)                            # [B, J]
    touched = pg * P < (L + n)[:, None]
    page = torch.gather(s["table"].long(), 1, pg.clamp(max=s["table"].shape[1] - 1))
    row = pg[..., None] * P + torch.arange(P, device=DEV)                         # [B, J, P]
    fresh = (row >= L[:, None, None]) & (row < (L + n)[:, None, None])
    token = (begin[:, None, None] + row - L[:, None, None]).clamp(0, x.shape[0] - 1)
    new = torch.where(fresh[..., None, None], x[token], 0.0).transpose(2, 3)      # [B, J, H, P, dh]
    pool = _bits(s[name])[0]
    held = pool[page.clamp(min=0)].view(s[name].dtype)
    fresh = fresh[:, :, None, :, None]
    if c["cache"] in QMAX:
        older = (row < L[:, None, None])[:, :, None, :, None]
        scale = s[name + "_scale"][0]
        was = torch.where((pg * P < L[:, None])[..., None], scale[page.clamp(min=0)], 0.0)
        now = torch.maximum(was, new.abs().amax((-2, -1)) / torch.full((), QMAX[c["cache"]], device=DEV))
        unit = torch.where(now > 0, now, 1.0).double()[..., None, None]
        again = _codes(c, held.float().double() * (was.double()[..., None, None] / unit))
        code = _codes(c, new.double() / unit)
        out = torch.where(fresh, _bits(code), torch.where(older, _bits(again), _bits(held)))
        scale[page[touched]] = now[touched]
    else:
        out = torch.where(fresh, new.to(torch.bfloat16), held)
    pool[page[touched]] = out[touched]


def _values(s, name, page):
    """Pages of any shape [...] as float32 [..., H, P, dh]."""
    x = _bits(s[name])[0][page].view(s[name].dtype).float()
    return x if s[name + "_scale"] is None else x * s[name + "_scale"][0][page][..., None, None]


def _read(s, name, first, n):
    """Rows first .. first + n - 1 (first: a page's) of every sequence as BF16 [B, H, n, dh]; rows without a page are zeros."""
    c = s["case"]
    P = c["page"]
    j = first.long()[:, None] // P + torch.arange((n + P - 1) // P, device=DEV)
    W = s["table"].shape[1]
    page = torch.where(j < W, torch.gather(s["table"].long(), 1, j.clamp(max=W - 1)), -1)
    x = torch.where((page >= 0)[..., None, None, None], _values(s, name, page.clamp(min=0)), 0.0)
    return x.transpose(1, 2).flatten(2, 3)[:, :, :n].to(torch.bfloat16)


def _append_plain(s):
    c, d = s["case"], s["rope"]
    b, i, _, _ = _tokens(s)
    angle = (s["len"].double()[b] + i)[:, None] * _frequencies(c, d, DEV)
    cos, sin = ((f(angle) * d["mscale"]).float()[:, None] for f in (torch.cos, torch.sin))
    _store(s, "kc", _rotate(c, s["k"].float(), cos, sin))
    _store(s, "vc", s["v"].float())
    q = _rotate(c, s["q"].float(), cos, sin)
    n = _read_rows(c)
    return {"q": q.to(TYPES[c["act"]]), "k": _read(s, "kc", s["first"], n), "v": _read(s, "vc", s["first"], n)}


def _attn_plain(s):
    c = s["case"]
    B, T, H, dh, P = c["batch"], c["T"], c["hkv"], c["dh"], c["page"]
    G = c["hq"] // H
    b, i, n, begin = _tokens(s)
    page = s["table"].long().clamp(min=0)
    R = page.shape[1] * P
    at = begin[:, None] + torch.arange(T, device=DEV)                             # padded to T tokens per sequence
    q = s["q"].float()[at.clamp(max=s["q"].shape[0] - 1)]
    q = q.reshape(B, T, H, G, dh).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, dh)
    k = _values(s, "kc", page).transpose(1, 2).reshape(B, H, R, dh)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(dh)
    del k
    hidden = torch.arange(R, device=DEV) > (s["len"].long()[:, None] + torch.arange(T, device=DEV))[..., None]     # [B, T, R]
    score = score.reshape(B, H, T, G, R).masked_fill_(hidden[:, None, :, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    del score
    total = p.sum(-1, keepdim=True)
    v = _values(s, "vc", page).transpose(1, 2).reshape(B, H, R, dh)
    o = torch.matmul(p.reshape(B, H, T * G, R), v).reshape(B, H, T, G, dh) / total
    return o.permute(0, 2, 1, 3, 4).reshape(B, T, c["hq"], dh)[b, i].to(TYPES[c["act"]])


def _score_plain(s):
    c = s["case"]
    V, K = c["vocab"], c["top"]
    x = s["logits"].float()
    token = s["tokens"].long()
    there = (token >= 0) & (token < V)
    token = token.clamp(0, V - 1)[:, None]
    top = x.amax(-1, keepdim=True)
    z = (x - top) / c["temperature"]
    w = torch.exp(z)
    total = w.sum(-1, dtype=torch.float64)
    entropy = torch.log(total) - (w * z).sum(-1, dtype=torch.float64) / total
    del w
    logprob = torch.where(there, torch.gather(z, 1, token)[:, 0].double() - torch.log(total), 0.0)
    mine = torch.gather(x, 1, token)
    ids = torch.arange(V, device=DEV)
    rank = torch.where(there, ((x > mine) | ((x == mine) & (ids < token))).sum(-1), -1)
    # the lowest id first where logits are equal: pairs of a logit, as a number that keeps its order, and an id
    order = (x + 0.0).view(torch.int32).long()
    order = torch.where(order < 0, -(order & 0x7fffffff), order)
    best = V - 1 - (torch.topk((order << 32) + (V - 1 - ids), min(K, V)).values & 0xffffffff)
    missing = K - best.shape[1]
    ids_out = torch.cat([best, best.new_full((best.shape[0], missing), -1)], 1)
    lp = torch.gather(z, 1, best).double() - torch.log(total)[:, None]
    lp = torch.cat([lp, lp.new_full((lp.shape[0], missing), -math.inf)], 1)
    row = torch.arange(c["rows"], device=DEV)
    inside = (row >= s["start"][:-1, None]) & (row < s["start"][1:, None]) & there               # [S, R]
    count = inside.sum(-1)
    mean = torch.where(inside, logprob, 0.0).sum(-1) / count.clamp(min=1)
    return {"logprob": logprob.float(), "entropy": entropy.float(), "rank": rank.to(torch.int32), "top_ids": ids_out.to(torch.int32),
            "top_logprobs": lp.float(), "mean": mean.float()}


# ----------------------------------------------------------------------------------- what a pass costs

def work(case):
    size = {"bf16": 2, "f32": 4, "int8": 1, "e4m3": 1}
    if case["kind"] == "score":
        n = float(case["rows"] * case["vocab"])
        return {"bytes": n * size[case["logits"]] + case["rows"] * (16.0 + 8 * case["top"]), "flops": 5 * n}
    lens, counts = _lens(case), _counts(case)
    N, P = sum(counts), case["page"]
    row = 2 * case["hkv"] * case["dh"] * size[case["cache"]]
    scales = 2 * case["hkv"] * 4 if case["cache"] in QMAX else 0
    pages = sum((n + c + P - 1) // P for n, c in zip(lens, counts))
    if case["kind"] == "append":
        acts = (2 * case["hq"] + 2 * case["hkv"]) * case["dh"] * size[case["act"]]
        touched = sum((n + c + P - 1) // P - n // P for n, c in zip(lens, counts))
        read = sum(c + n % P for n, c in zip(lens, counts))
        return {"bytes": float(N * (acts + row) + read * (row + 2 * case["hkv"] * case["dh"] * 2) + 2 * touched * scales),
                "flops": N * (case["hq"] + 2.0 * case["hkv"]) * case["dh"] * 3}
    shared = min(case["shared"], min(n // P for n in lens)) * (case["batch"] - 1)
    acts = 2 * N * case["hq"] * case["dh"] * size[case["act"]]
    seen = sum(c * n + c * (c + 1) // 2 for n, c in zip(lens, counts))
    return {"bytes": float((sum(lens) + N - shared * P) * row + (pages - shared) * scales + acts),
            "flops": 4.0 * seen * case["hq"] * case["dh"]}


# ----------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "score": _exact_score}[case["kind"]](case, s)


def _exact_score(case, s):
    V, K, T = case["vocab"], case["top"], case["temperature"]
    cols = {n: [] for n in ("logprob", "entropy", "rank", "top_ids", "top_logprobs")}
    for a in range(0, case["rows"], 64):
        x = s["logits"][a:a + 64].double()
        t = s["tokens"][a:a + 64].long()
        lp = torch.log_softmax(x / T, -1)
        cols["entropy"].append(-(lp.exp() * lp).sum(-1))
        sorted_ids = torch.sort(x, dim=-1, descending=True, stable=True).indices
        known = (t >= 0) & (t < V)
        place = (sorted_ids == t[:, None]).double().argmax(-1)
        cols["rank"].append(torch.where(known, place, -1).to(torch.int32))
        cols["logprob"].append(torch.where(known, lp.gather(1, t.clamp(0, V - 1)[:, None])[:, 0], 0.0))
        best = sorted_ids[:, :K]
        pad = (0, K - best.shape[1])
        cols["top_ids"].append(torch.nn.functional.pad(best, pad, value=-1).to(torch.int32))
        cols["top_logprobs"].append(torch.nn.functional.pad(lp.gather(1, best), pad, value=-math.inf))
    out = {n: torch.cat(v) for n, v in cols.items()}
    at, known, mean = s["start"].tolist(), (s["tokens"] >= 0) & (s["tokens"] < V), []
    for a, b in zip(at, at[1:]):
        mine = out["logprob"][a:b][known[a:b]]
        mean.append(mine.mean() if len(mine) else torch.zeros((), dtype=torch.float64, device=DEV))
    out["mean"] = torch.stack(mean)
    return out


def _rows_of(case, s, name, b, n):
    """Rows 0 .. n - 1 of a sequence in 64 bits [n, H, dh]."""
    P = case["page"]
    ids = s["table"][b, :(n + P - 1) // P].long()
    x = s[name][0].view(torch.uint8)[ids].view(s[name].dtype).double()
    if case["cache"] in QMAX:
        x = x * s[name + "_scale"][0][ids].double()[:, :, None, None]
    return x.permute(0, 2, 1, 3).reshape(-1, case["hkv"], case["dh"])[:n]


def _exact_attn(case, s):
    lens, counts, H, dh = _lens(case), _counts(case), case["hkv"], case["dh"]
    G = case["hq"] // H
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    t0 = 0
    for b, (L, n) in enumerate(zip(lens, counts)):
        k, v = _rows_of(case, s, "kc", b, L + n), _rows_of(case, s, "vc", b, L + n)
        for a in range(0, n, 512):
            m = min(512, n - a)
            end = L + a + m
            hide = torch.ones((m, end), dtype=torch.bool, device=DEV).triu(L + a + 1)
            for h in range(H):
                x = s["q"][t0 + a:t0 + a + m, h * G:(h + 1) * G].double()
                z = (x.reshape(m * G, dh) @ k[:end, h].T * dh ** -0.5).reshape(m, G, end).masked_fill(hide[:, None], -math.inf)
                p = torch.softmax(z, -1).reshape(m * G, end)
                out[t0 + a:t0 + a + m, h * G:(h + 1) * G] = (p @ v[:end, h]).reshape(m, G, dh)
        t0 += n
    return out


def _exact_append(case, s):
    lens, counts, H, dh, P, n = _lens(case), _counts(case), case["hkv"], case["dh"], case["page"], case["rot"]
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
    pos = torch.cat([torch.arange(L, L + c, dtype=torch.float64, device=DEV) for L, c in zip(lens, counts)])
    turn = torch.polar(torch.full((), d["mscale"], dtype=torch.float64, device=DEV), pos[:, None] * torch.tensor(freq, dtype=torch.float64, device=DEV))

    def turned(x):
        x = x.double().clone()
        first, second = (slice(0, n // 2), slice(n // 2, n)) if case["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
        z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
        x[..., first], x[..., second] = z.real, z.imag
        return x

    def rounded(x):
        return torch.round(x) if case["cache"] == "int8" else x.float().to(torch.float8_e4m3fn).double()

    rows = _read_rows(case)

    def held(name, x):
        out = torch.zeros((case["batch"], H, rows, dh), dtype=torch.float64, device=DEV)
        t0 = 0
        for b, (L, c) in enumerate(zip(lens, counts)):
            base = L // P * P
            pages = s["table"][b, base // P:].tolist()
            for j, page in enumerate(pages):           # a page's rows: older, new, and what lies behind them
                lo = base + j * P
                if page < 0 or lo >= base + rows:
                    break
                code = s[name][0, page].double()
                a, z = max(L, lo) - lo, min(L + c, lo + P) - lo
                new = x[t0 + lo + a - L:t0 + lo + z - L].transpose(0, 1) if z > a else None
                if case["cache"] == "bf16":
                    if new is not None:
                        code[:, a:z] = new
                else:
                    scale = s[name + "_scale"][0, page].double()[:, None, None]
                    if new is not None:
                        was = scale if lo < L else torch.zeros_like(scale)
                        scale = torch.maximum(was, new.abs().amax((1, 2))[:, None, None] / QMAX[case["cache"]])
                        scale[scale == 0] = 1.0
                        code[:, :a] = rounded(code[:, :a] * (was / scale))
                        code[:, a:z] = rounded(new / scale)
                    code = code * scale
                take = min(P, base + rows - lo)
                out[b, :, lo - base:lo - base + take] = code[:, :take]
            t0 += c
        return out

    return {"q": turned(s["q"]), "k": held("kc", turned(s["k"])), "v": held("vc", s["v"].double())}
