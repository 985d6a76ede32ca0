"""Host-side refusals of the drafted-token entry points: wrong types, shapes, alignments and
workspaces are rejected before any GPU work (the addresses are never dereferenced)."""
import ctypes as C

import pytest
import torch

from paper_2609_29499_amd import binding as B
from paper_2609_29499_amd import session as S

FAKE = 1 << 20


def cache(**kw):
    c = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, len=FAKE, type=B.INT8, n_layers=2, batch=3, n_kv_heads=4,
             max_seq=100, head_dim=128, plan_sig=0)
    c.update(kw)
    return B.tasp_seq_cache(*[c[n] for n, _ in B.tasp_seq_cache._fields_])


def rows(p=FAKE, seq=8192, token=1024, head=128):
    return B.tasp_rows(p, seq, token, head)


def rope(**kw):
    r = dict(layout=0, rot_dim=128, scaling=0, orig_len=8192, theta=500000.0, factor=8.0, low=1.0, high=4.0, mscale=1.0)
    r.update(kw)
    return B.tasp_rope(*[r[n] for n, _ in B.tasp_rope._fields_])


def refused(status, f, *a):
    B.load()
    with pytest.raises(B.TaspError) as e:
        f(*a)
    assert B.STATUS[e.value.status] == status, e.value


BAD_CACHES = [
    (dict(type=B.F32), "TASP_ERR_INVALID_ARG"), (dict(type=7), "TASP_ERR_INVALID_ARG"),
    (dict(head_dim=96), "TASP_ERR_SHAPE"), (dict(batch=0), "TASP_ERR_SHAPE"), (dict(batch=257), "TASP_ERR_SHAPE"),
    (dict(n_kv_heads=65), "TASP_ERR_SHAPE"), (dict(max_seq=0), "TASP_ERR_SHAPE"), (dict(n_layers=0), "TASP_ERR_SHAPE"),
    (dict(max_seq=1 << 23), "TASP_ERR_SHAPE"), (dict(k=None), "TASP_ERR_INVALID_ARG"), (dict(v=FAKE + 8), "TASP_ERR_INVALID_ARG"),
    (dict(len=None), "TASP_ERR_INVALID_ARG"), (dict(len=FAKE + 2), "TASP_ERR_INVALID_ARG"),
    (dict(k_scale=None), "TASP_ERR_INVALID_ARG"), (dict(v_scale=FAKE + 1), "TASP_ERR_INVALID_ARG"),
]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_bad_caches(kw, status):
    c = cache(**kw)
    refused(status, B.tasp_seq_append, c, 0, None, None, 1, B.BF16, None, rows(), rows(), 0, None, None)
    refused(status, B.tasp_seq_read, c, 0, None, 1, B.BF16, rows(), rows(), None)
    refused(status, B.tasp_tree_attention, c, 0, None, 1, B.BF16, rows(), 8, 0.1, 100, rows(), FAKE, 1 << 40, None)
    refused(status, B.tasp_seq_commit, c, FAKE, FAKE, 4, FAKE, None)


def test_append_refusals():
    ok = [cache(), 1, rope(), None, 5, B.BF16, rows(), rows(), rows(), 8, rows(), None]

    def bad(status, **at):
        a = list(ok)
        for i, v in at.items():
            a[int(i[1:])] = v
        refused(status, B.tasp_seq_append, *a)

    bad("TASP_ERR_SHAPE", _1=2)
    bad("TASP_ERR_SHAPE", _1=-1)
    bad("TASP_ERR_SHAPE", _4=0)
    bad("TASP_ERR_SHAPE", _4=101)                              # more tokens than rows
    bad("TASP_ERR_SHAPE", _3=FAKE, _4=65)                      # a tree of more than 64
    bad("TASP_ERR_INVALID_ARG", _3=FAKE + 1)
    bad("TASP_ERR_INVALID_ARG", _5=B.INT8)
    for i in ("_6", "_7", "_8", "_10"):
        bad("TASP_ERR_INVALID_ARG", **{i: None})
        bad("TASP_ERR_INVALID_ARG", **{i: rows(p=FAKE + 8)})
        bad("TASP_ERR_INVALID_ARG", **{i: rows(token=1028)})   # BF16 rows 8-byte aligned
    bad("TASP_ERR_INVALID_ARG", _9=0)                          # queries without heads
    bad("TASP_ERR_SHAPE", _9=513)
    for kw, st in ((dict(layout=2), "TASP_ERR_INVALID_ARG"), (dict(rot_dim=8), "TASP_ERR_SHAPE"),
                   (dict(rot_dim=144), "TASP_ERR_SHAPE"), (dict(scaling=4), "TASP_ERR_INVALID_ARG"),
                   (dict(theta=1.0), "TASP_ERR_INVALID_ARG"), (dict(theta=float("nan")), "TASP_ERR_INVALID_ARG"),
                   (dict(mscale=float("inf")), "TASP_ERR_INVALID_ARG"), (dict(scaling=1, factor=0.0), "TASP_ERR_INVALID_ARG"),
                   (dict(scaling=2, low=4.0), "TASP_ERR_INVALID_ARG"), (dict(scaling=3, orig_len=0), "TASP_ERR_INVALID_ARG")):
        bad(st, _2=rope(**kw))


def test_read_and_commit_refusals():
    c = cache()
    refused("TASP_ERR_SHAPE", B.tasp_seq_read, c, 0, None, 0, B.BF16, rows(), rows(), None)
    refused("TASP_ERR_INVALID_ARG", B.tasp_seq_read, c, 0, FAKE + 2, 1, B.BF16, rows(), rows(), None)
    refused("TASP_ERR_INVALID_ARG", B.tasp_seq_read, c, 0, None, 1, B.E4M3, rows(), rows(), None)
    refused("TASP_ERR_INVALID_ARG", B.tasp_seq_read, c, 0, None, 1, B.F32, rows(), rows(head=130), None)
    for T in (0, 65):
        refused("TASP_ERR_SHAPE", B.tasp_seq_commit, c, FAKE, FAKE, T, FAKE, None)
    for a in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None), (FAKE + 1, FAKE, FAKE)):
        refused("TASP_ERR_INVALID_ARG", B.tasp_seq_commit, c, a[0], a[1], 4, a[2], None)


def test_attention_refusals_and_workspace():
    B.load()
    c = cache(batch=1, max_seq=5000)
    nb = B.tasp_tree_attention_workspace_bytes(c, 8, 4, 5000)
    assert nb > 0 and B.tasp_tree_attention_workspace_bytes(c, 8, 4, 0) == 0     # short ones need none
    ok = [c, 0, None, 4, B.BF16, rows(), 8, 0.1, 5000, rows(), FAKE, nb, None]

    def bad(status, **at):
        a = list(ok)
        for i, v in at.items():
            a[int(i[1:])] = v
        refused(status, B.tasp_tree_attention, *a)

    for T in (0, 65):
        bad("TASP_ERR_SHAPE", _3=T)
        refused("TASP_ERR_SHAPE", B.tasp_tree_attention_workspace_bytes, c, 8, T, 100)
    for hq in (0, 6, 36):
        bad("TASP_ERR_SHAPE", _6=hq)
    for m in (-1, 5001):
        bad("TASP_ERR_SHAPE", _8=m)
    for x in (0.0, -1.0, float("nan"), float("inf")):
        bad("TASP_ERR_INVALID_ARG", _7=x)
    for i in ("_5", "_9"):
        bad("TASP_ERR_INVALID_ARG", **{i: None})
        bad("TASP_ERR_INVALID_ARG", **{i: rows(p=FAKE + 4)})
    bad("TASP_ERR_WORKSPACE", _11=nb - 1)
    bad("TASP_ERR_WORKSPACE", _10=FAKE + 16)
    bad("TASP_ERR_INVALID_ARG", _10=None)


def test_verify_refusals():
    B.load()
    nb = B.tasp_verify_workspace_bytes(2, 5, 1000)
    ok = [FAKE, FAKE, FAKE, None, None, 2, 5, 1000, 1.0, FAKE, FAKE, FAKE, FAKE, nb, None]

    def bad(status, **at):
        a = list(ok)
        for i, v in at.items():
            a[int(i[1:])] = v
        refused(status, B.tasp_verify, *a)

    for i in (0, 1, 2, 9, 10, 11, 12):
        bad("TASP_ERR_INVALID_ARG", **{f"_{i}": None})
        if i != 12:
            bad("TASP_ERR_INVALID_ARG", **{f"_{i}": FAKE + 2})
    for i, vs in ((5, (0, 257)), (6, (0, 65)), (7, (0, (1 << 24) + 1))):
        for v in vs:
            bad("TASP_ERR_SHAPE", **{f"_{i}": v})
            refused("TASP_ERR_SHAPE", B.tasp_verify_workspace_bytes, *[v if i == j else x for j, x in ((5, 2), (6, 5), (7, 1000))])
    for t in (-0.5, float("nan"), float("inf"), 1e-310):
        bad("TASP_ERR_INVALID_ARG", _8=t)
    bad("TASP_ERR_INVALID_ARG", _3=FAKE, _4=FAKE)              # draft logits with a tree
    bad("TASP_ERR_WORKSPACE", _13=nb - 1)
    bad("TASP_ERR_WORKSPACE", _12=FAKE + 64)


def test_session_refuses_tensors_before_the_library():
    k = torch.zeros((1, 2, 2, 8, 64), dtype=torch.bfloat16)
    ln = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        S.SeqCache(k, k.clone(), ln)
    with pytest.raises(ValueError, match="bfloat16, int8"):
        S.SeqCache(k.float(), k.float(), ln)
    with pytest.raises(ValueError):
        S._ptr(ln, (3,), torch.int32, "len")
    with pytest.raises(ValueError):
        S._rows(k[0].transpose(2, 3), (2, 2, 64, 8), torch.bfloat16, "q")
    r = B.tasp_rows.from_buffer_copy(S._rows(k[0], (2, 2, 8, 64), torch.bfloat16, "k", 2, 1))
    assert (r.p, r.seq, r.token, r.head) == (k.data_ptr(), 1024, 64, 512)
    assert B.tasp_rows.from_buffer_copy(S._rows(k[0, :, :1], (2, 1, 8, 64), torch.bfloat16, "k")).token == 0
    assert C.sizeof(B.tasp_rows) == 32 and C.sizeof(B.tasp_seq_cache) == 72 and C.sizeof(B.tasp_rope) == 56


@pytest.mark.parametrize("t", [1e-31, 1e31, -1e-30, 5e-324])
def test_temperatures_out_of_range(t):
    B.load()
    nb = B.tasp_verify_workspace_bytes(1, 1, 100)
    refused("TASP_ERR_INVALID_ARG", B.tasp_verify, FAKE, FAKE, FAKE, None, None, 1, 1, 100, t, FAKE, FAKE, FAKE, FAKE, nb, None)


def test_types_that_are_no_activations():
    k = torch.zeros((1, 2, 2, 8, 64), dtype=torch.float16)
    with pytest.raises(ValueError, match="float16"):
        S._SEQ_TYPES[k.dtype]


def test_plan_steps_refuse_no_plan():
    c = cache()
    refused("TASP_ERR_INVALID_ARG", B.tasp_seq_bind, None, c)
    refused("TASP_ERR_INVALID_ARG", B.tasp_tree_step_workspace_bytes, None, c, 4, 100)
    refused("TASP_ERR_INVALID_ARG", B.tasp_tree_forward, None, FAKE, None, 4, c, 100, FAKE, FAKE, 1 << 30, None)
    refused("TASP_ERR_INVALID_ARG", B.tasp_tree_step, None, FAKE, FAKE, FAKE, None, FAKE, None, 1.0, 4, 100, c, FAKE, FAKE,
            FAKE, FAKE, FAKE, FAKE, 1 << 30, None)
