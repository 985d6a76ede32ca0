"""Attention of drafted nodes over cached rows and ancestors against the float64 oracle.

Tolerance of one output: with A = sum of p |v| over the rows seen, n their number,
  scores: a float32 dot product of dh exact products, |error| <= (dh + 4) 2^-24 scale sum |q_i k_i| = d, which
  moves p by a factor within exp(2 d);
  exp2 and the rescaling by powers: 2^-21; P in two BF16 terms 2^-16, in three 2^-24; over rows in 8 bits with more
  than 32 BF16 query rows P is one FP16 term: half a step 2^-11, and where P times the row's scale falls below 2^-18 of the largest scale M,
  a subnormal's half step 2^-25 in units of 2^-4 M or less: n 2^-29 max |v| together; float32 sums n 2^-24;
  the output's rounding 2^-8 of the value in BF16, 2^-24 in float32.
|error| <= A (2 d + 2^-21 + 2^-11, 2^-16 or 2^-24 + n 2^-24) + (n 2^-29 max |v|) + |o| 2^-8 or 2^-24."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2609_29499_amd import session as S
from tests.seq_case import DTYPES, flush, gen, randn, random_parents, typed_cache

pytestmark = pytest.mark.gpu


def check(got, q, kv, vv, lens, parent, S_, act, scale, nodes=None, kind="bf16"):
    """got [B][T][Hq][dh] against the oracle, every node or the given ones."""
    Bn, T, hq, dh = q.shape
    H = kv.shape[1]
    half = kind != "bf16" and act == "bf16" and T * (hq // H) > 32
    worst = 0.0
    for b in range(Bn):
        ln = O.lines(None if parent is None else parent[b].tolist(), T, S_ - lens[b]) if 0 <= lens[b] <= S_ else [None] * T
        for t in range(T) if nodes is None else nodes:
            if ln[t] is None:
                assert not got[b, t].any(), (b, t)
                continue
            seen = list(range(lens[b])) + [lens[b] + j for j in ln[t]]
            for h in range(hq):
                k, v = kv[b, h // (hq // H)], vv[b, h // (hq // H)]
                o, A = O.attention(q[b, t, h], k, v, seen, scale)
                d = (dh + 4) * 2.0 ** -24 * scale * np.max(np.abs(k[seen]) @ np.abs(q[b, t, h]))
                tol = A * (2 * d + 2.0 ** -21 + (2.0 ** -11 if half else 2.0 ** -16 if act == "bf16" else 2.0 ** -24) + len(seen) * 2.0 ** -24)
                tol = tol + half * len(seen) * 2.0 ** -29 * np.max(np.abs(v[seen]))
                tol = tol + np.abs(o) * (2.0 ** -8 if act == "bf16" else 2.0 ** -24)
                err = np.abs(got[b, t, h] - o)
                worst = max(worst, float(np.max(np.divide(err, tol, out=np.zeros_like(err), where=tol > 0))))
                assert np.all(err <= tol), (b, t, h, float(np.max(err / tol)))
    flush(f"   worst share of the tolerance {worst:.3f}")


CASES = [
    # lens, room behind, T, hq, hkv, dh, cache, act, tree
    ([0], 0, 1, 4, 4, 64, "bf16", "bf16", False),
    ([1], 3, 1, 8, 1, 128, "int8", "bf16", False),
    ([0, 5, 31], 0, 3, 6, 3, 64, "int8", "bf16", True),
    ([32, 31, 33, 0], 2, 5, 8, 2, 128, "e4m3", "bf16", True),
    ([127, 128, 129], 0, 16, 4, 1, 128, "bf16", "bf16", True),
    ([300, 0, 17], 5, 64, 8, 1, 128, "int8", "bf16", True),
    ([77, 500], 0, 33, 9, 3, 64, "bf16", "f32", True),
    ([600], 0, 7, 28, 4, 128, "e4m3", "f32", False),
    ([2000, 3, 900, 0, 1500], 1, 2, 16, 2, 64, "e4m3", "bf16", True),
    ([4100], 0, 1, 4, 1, 64, "int8", "f32", False),
    ([-3, 50, 64], 0, 4, 4, 2, 64, "int8", "bf16", False),          # a length out of range
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_tree_attention(case):
    lens, room, T, hq, H, dh, kind, act, tree = CASES[case]
    flush(f"case attention {CASES[case]}")
    S_ = max(lens) + T + room if case != 10 else 66                 # (the last case: two nodes do not fit)
    c, kv, vv = typed_cache(lens, H, S_, dh, kind, case)
    parent = random_parents(len(lens), T, case) if tree else None
    q = randn((len(lens), T, hq, dh), DTYPES[act], 100 + case)
    got = S.tree_attention(c, 0, q.cuda(), None if parent is None else parent.cuda())
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), kv[0], vv[0], lens, parent, S_, act, dh ** -0.5, kind=kind)


@pytest.mark.parametrize("kind,T,hq,dh", [("bf16", 3, 4, 128), ("int8", 3, 4, 128), ("e4m3", 9, 8, 64),
                                          ("int8", 12, 8, 128), ("bf16", 20, 8, 64), ("e4m3", 33, 8, 128)])
def test_long_contexts_in_many_chunks(kind, T, hq, dh):
    """Ragged sequences over several chunks, a hint of the length that is too small, strided q and out."""
    lens = [20000, 700, 0, 9001]
    flush(f"case long {kind} {T} {hq} {dh}")
    H = 2
    c, kv, vv = typed_cache(lens, H, 20040, dh, kind, 7)
    parent = random_parents(4, T, 7, absent=False)
    wide = torch.zeros((4, T, 3, hq, dh), dtype=torch.bfloat16, device="cuda")
    q = randn((4, T, hq, dh), torch.bfloat16, 8)
    wide[:, :, 1] = q.cuda()
    out = torch.full((4, T, hq + 1, dh), 5.0, dtype=torch.bfloat16, device="cuda")
    outs = []
    for hint in (20000, 4000, 100):
        S.tree_attention(c, 0, wide[:, :, 1], parent.cuda(), max_len=hint, out=out[:, :, :hq])
        torch.cuda.synchronize()
        check(out[:, :, :hq].double().cpu().numpy(), q.double().numpy(), kv[0], vv[0], lens, parent, 20040, "bf16", dh ** -0.5, sorted({0, T // 2, T - 1}), kind=kind)
        assert torch.all(out[:, :, hq] == 5.0)
        again = S.tree_attention(c, 0, wide[:, :, 1], parent.cuda(), max_len=hint)
        torch.cuda.synchronize()
        assert torch.equal(again, out[:, :, :hq])                   # the same call gives the same bits
        outs.append(again)


def test_layers_behind_32_bit_offsets():
    """The last layer of a cache of more than 2^32 bytes."""
    flush("case far layer")
    L, H, S_, dh = 5, 8, 1 << 20, 128
    k = torch.zeros((L, 1, H, S_, dh), dtype=torch.int8, device="cuda")
    assert k.numel() > 1 << 32
    v, sc = torch.zeros_like(k), torch.full((L, 1, H, S_), 0.01, device="cuda")
    lens = S_ - 2
    c = S.SeqCache(k, v, torch.tensor([lens], dtype=torch.int32, device="cuda"), sc, sc)
    x = randn((1, 2, H, dh), torch.bfloat16, 9).cuda()
    S.seq_append(c, L - 1, None, x, x)
    # node 1 scores its own row far above the zeros': its value comes out
    q = x * 40.0
    out = S.tree_attention(c, L - 1, q, torch.tensor([[-1, -1]], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    step = x.float().abs().amax(-1, keepdim=True) / 127
    assert torch.all((out.float() - x.float()).abs() <= step * 0.51 + x.float().abs() * 2.0 ** -7)
    assert not c.k[:L - 1].any() and not c.k[L - 1, 0, :, :lens].any()


@pytest.mark.parametrize("hq", [4, 16])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
def test_unseen_rows_reach_nothing(kind, hq):
    """Infinities and NaN in rows of other branches, of absent nodes and behind the nodes."""
    flush(f"case unseen {kind} {hq}")
    lens, T, dh = [40, 0], 6, 64
    S_ = 60
    c, kv, vv = typed_cache(lens, 2, S_, dh, kind, 10)
    parent = torch.tensor([[-1, 0, 0, 1, 2, -2], [-1, 0, 0, 1, 2, -2]], dtype=torch.int32)
    q = randn((2, T, hq, dh), torch.bfloat16, 11)
    clean = S.tree_attention(c, 0, q.cuda(), parent.cuda())
    for b in range(2):
        for r, what in ((2, math.nan), (5, math.inf), (7, math.nan)):      # node 2, an absent node, behind the tree
            if kind == "bf16":
                c.k[0, b, :, lens[b] + r] = what
                c.v[0, b, :, lens[b] + r, ::5] = what
                c.v[0, b, :, lens[b] + r, 1::5] = -math.inf
            else:
                c.k_scale[0, b, :, lens[b] + r] = math.nan
                c.v_scale[0, b, :, lens[b] + r] = math.nan
            if kind == "e4m3":
                c.v.view(torch.uint8)[0, b, :, lens[b] + r] = 0x7f         # NaN codes
    got = S.tree_attention(c, 0, q.cuda(), parent.cuda())
    torch.cuda.synchronize()
    for t in (0, 1, 3, 5):                                                 # nodes that do not see node 2
        assert torch.equal(got[:, t], clean[:, t]), t
    assert torch.isnan(got[:, 2]).any(-1).all() and torch.isnan(got[:, 4]).any(-1).all()


@pytest.mark.parametrize("T", [3, 17])
def test_visible_infinities_stay_in_their_dimensions(T):
    flush(f"case visible infinities {T}")
    c, kv, vv = typed_cache([10], 1, 30, 64, "bf16", 12)
    q = randn((1, T, 2, 64), torch.bfloat16, 13).cuda()
    parent = torch.tensor([[-1] + [0] * (T - 1)], dtype=torch.int32, device="cuda")
    clean = S.tree_attention(c, 0, q, parent)
    c.v[0, 0, 0, 11, 3], c.v[0, 0, 0, 11, 4], c.v[0, 0, 0, 11, 5] = math.inf, -math.inf, math.nan
    c.v[0, 0, 0, 10, 4] = math.inf
    c.v[0, 0, 0, 6, 8] = math.nan                                       # a cached row, next to the tree's
    got = S.tree_attention(c, 0, q, parent).float()
    torch.cuda.synchronize()
    assert torch.all(got[0, 1, :, 3] == math.inf) and torch.isnan(got[0, 1, :, 4:6]).all()   # node 1: its own row and node 0's
    assert torch.all(got[0, 0, :, 4] == math.inf) and torch.all(got[0, 2, :, 4] == math.inf)
    assert torch.isnan(got[0, :, :, 8]).all()
    rest = [d for d in range(64) if d not in (3, 4, 5, 8)]
    assert torch.equal(got[0][:, :, rest], clean.float()[0][:, :, rest])


def test_large_scores_and_one_step_rises():
    """Scores that grow along the cache by far more than one power of two per step, and a scale of its own."""
    flush("case rising scores")
    c, kv, vv = typed_cache([700], 1, 704, 64, "bf16", 14)
    ramp = torch.linspace(0, 1, 704)[:, None] * torch.ones(64)
    c.k[0, 0, 0] = ramp.to(torch.bfloat16).cuda()
    q = torch.full((1, 2, 2, 64), 1.0, dtype=torch.bfloat16)
    q[0, 1] = -1.0
    got = S.tree_attention(c, 0, q.cuda(), scale=30.0)
    torch.cuda.synchronize()
    k64 = c.k.double().cpu().numpy()
    g = got.double().cpu().numpy()
    check(g, q.double().numpy(), k64[0], vv[0], [700], None, 704, "bf16", 30.0)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("dh", [64, 128])
def test_every_block_of_query_rows(dh, kind, act):
    """1, 2, 3 .. 4, 5 .. 8 and more tiles of 16 query rows (every kernel), in one chunk and in several."""
    flush(f"case blocks {dh} {kind} {act}")
    for T, hq, lens in ((3, 4, [70, 1]), (5, 6, [33, 400]), (9, 6, [90, 700]), (13, 8, [5, 311]), (23, 8, [64, 190])):
        S_ = max(lens) + T
        c, kv, vv = typed_cache(lens, 1, S_, dh, kind, T)
        parent = random_parents(2, T, T, absent=False)
        q = randn((2, T, hq, dh), DTYPES[act], 50 + T)
        got = S.tree_attention(c, 0, q.cuda(), parent.cuda())
        torch.cuda.synchronize()
        check(got.double().cpu().numpy(), q.double().numpy(), kv[0], vv[0], lens, parent, S_, act, dh ** -0.5, kind=kind)


@pytest.mark.parametrize("kind,act,dh", [("int8", "bf16", 128), ("bf16", "bf16", 64), ("e4m3", "f32", 64), ("bf16", "f32", 128)])
def test_wide_trees_of_a_ragged_batch(kind, act, dh):
    """Few workgroups per sequence: they take pieces of neighbouring sequences, of which some are empty, one row, out
    of range or longer than expected."""
    flush(f"case ragged {kind} {act} {dh}")
    lens, T, H = [900, 0, 1, 610, -2, 33, 500, 64], 64, 8 if act == "bf16" else 4
    hq = 8 * H
    c, kv, vv = typed_cache(lens, H, 964, dh, kind, 11)
    parent = random_parents(len(lens), T, 11)
    q = randn((len(lens), T, hq, dh), DTYPES[act], 12)
    for max_len in (900, 640):
        got = S.tree_attention(c, 0, q.cuda(), parent.cuda(), max_len=max_len)
        torch.cuda.synchronize()
        check(got.double().cpu().numpy(), q.double().numpy(), kv[0], vv[0], lens, parent, 964, act, dh ** -0.5, nodes=[0, 17, 63], kind=kind)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed", "zeros"])
def test_scales_of_any_size(kind, order):
    """Values that grow or shrink by 40 powers of two along the cache, or are nothing but zeros, under wide trees."""
    flush(f"case scales {kind} {order}")
    lens, T, hq, dh = [500, 130], 12, 8, 64
    c, kv, vv = typed_cache(lens, 1, 520, dh, kind, 15)
    x = torch.linspace(-20, 20, 520)
    if order == "mixed":
        x = x[torch.randperm(520, generator=gen(16))]
    f = torch.zeros(520) if order == "zeros" else torch.exp2((x if order != "falling" else -x).round())
    c.v_scale.mul_(f.cuda())
    parent = random_parents(2, T, 15)
    q = randn((2, T, hq, dh), torch.bfloat16, 17)
    got = S.tree_attention(c, 0, q.cuda(), parent.cuda())
    torch.cuda.synchronize()
    values = np.asarray(vv[0]) * f.double().numpy()[:, None]
    check(got.double().cpu().numpy(), q.double().numpy(), kv[0], values, lens, parent, 520, "bf16", dh ** -0.5, kind=kind)
    if order == "zeros":
        assert not got.any()


def test_visible_scales_that_are_not_finite():
    """A cached row whose scale is infinite or NaN: its nodes' outputs are not finite, and others' stay what they are."""
    flush("case scales not finite")
    T, dh = 12, 64
    c, kv, vv = typed_cache([100, 100], 1, 120, dh, "int8", 18)
    q = randn((2, T, 8, dh), torch.bfloat16, 19).cuda()
    clean = S.tree_attention(c, 0, q)
    for what in (math.inf, math.nan):
        c.v_scale[0, 1, 0, 50] = what
        got = S.tree_attention(c, 0, q)
        torch.cuda.synchronize()
        assert torch.equal(got[0], clean[0]) and not torch.isfinite(got[1]).any()


def test_two_calls_at_once():
    """Two caches on two streams, a workspace of each call's own: what each gives alone."""
    flush("case two streams")
    runs = []
    for k in range(2):
        c, _, _ = typed_cache([1500, 700], 2, 1600, 128, "int8", 40 + k)
        runs.append((c, randn((2, 20, 8, 128), torch.bfloat16, 50 + k).cuda(), torch.cuda.Stream()))
    alone = [S.tree_attention(c, 0, q) for c, q, _ in runs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [S.tree_attention(c, 0, q, stream=s.cuda_stream) for c, q, s in runs]
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, alone))
