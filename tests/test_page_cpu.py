"""Host-side refusals of the paged-cache and token-score entry points: wrong types, shapes, alignments and
workspaces are rejected before any GPU work (the addresses are never dereferenced)."""
import ctypes as C

import pytest
import torch

from paper_2609_29499_amd import binding as B
from paper_2609_29499_amd import session as S

FAKE = 1 << 20


def cache(**kw):
    c = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, table=FAKE, len=FAKE, type=B.INT8, n_layers=2, n_pages=50, n_kv_heads=4,
             page_rows=32, head_dim=128, batch=3, max_pages=10, plan_sig=0)
    c.update(kw)
    return B.tasp_page_cache(*[c[n] for n, _ in B.tasp_page_cache._fields_])


def rows(p=FAKE, seq=0, token=1024, head=128):
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


def changed(ok, at):
    return [at.get(i, x) for i, x in enumerate(ok)]


BAD_CACHES = [
    (dict(type=B.F32), "TASP_ERR_INVALID_ARG"), (dict(type=7), "TASP_ERR_INVALID_ARG"), (dict(head_dim=96), "TASP_ERR_SHAPE"),
    (dict(batch=0), "TASP_ERR_SHAPE"), (dict(batch=257), "TASP_ERR_SHAPE"), (dict(n_kv_heads=65), "TASP_ERR_SHAPE"),
    (dict(n_kv_heads=0), "TASP_ERR_SHAPE"), (dict(n_pages=0), "TASP_ERR_SHAPE"), (dict(max_pages=0), "TASP_ERR_SHAPE"),
    (dict(n_layers=0), "TASP_ERR_SHAPE"), (dict(page_rows=8), "TASP_ERR_SHAPE"), (dict(page_rows=48), "TASP_ERR_SHAPE"),
    (dict(page_rows=256), "TASP_ERR_SHAPE"), (dict(page_rows=0), "TASP_ERR_SHAPE"), (dict(max_pages=(1 << 18) + 1), "TASP_ERR_SHAPE"),
    (dict(max_pages=(1 << 31) - 1), "TASP_ERR_SHAPE"), (dict(k=None), "TASP_ERR_INVALID_ARG"), (dict(v=FAKE + 8), "TASP_ERR_INVALID_ARG"),
    (dict(len=None), "TASP_ERR_INVALID_ARG"), (dict(len=FAKE + 2), "TASP_ERR_INVALID_ARG"), (dict(table=None), "TASP_ERR_INVALID_ARG"),
    (dict(table=FAKE + 2), "TASP_ERR_INVALID_ARG"), (dict(k_scale=None), "TASP_ERR_INVALID_ARG"), (dict(v_scale=FAKE + 1), "TASP_ERR_INVALID_ARG"),
]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_bad_caches(kw, status):
    c = cache(**kw)
    refused(status, B.tasp_page_append, c, 0, None, FAKE, 4, B.BF16, None, rows(), rows(), 0, None, None)
    refused(status, B.tasp_page_read, c, 0, None, 1, B.BF16, rows(), rows(), None)
    refused(status, B.tasp_page_attention, c, 0, FAKE, 4, B.BF16, rows(), 8, 0.1, 100, 2, rows(), FAKE, 1 << 40, None)


def test_append_refusals():
    ok = [cache(), 1, rope(), FAKE, 5, B.BF16, rows(), rows(), rows(), 8, rows(), None]

    def bad(status, **at):
        refused(status, B.tasp_page_append, *changed(ok, {int(k[1:]): v for k, v in at.items()}))

    bad("TASP_ERR_INVALID_ARG", _0=None)
    bad("TASP_ERR_SHAPE", _1=2)
    bad("TASP_ERR_SHAPE", _1=-1)
    for n in (0, -1, B.PAGE_MAX_TOKENS + 1):
        bad("TASP_ERR_SHAPE", _4=n)
    bad("TASP_ERR_SHAPE", _3=None)                     # five tokens of three sequences
    bad("TASP_ERR_INVALID_ARG", _3=FAKE + 2)
    bad("TASP_ERR_INVALID_ARG", _5=B.INT8)
    for i in (6, 7, 8, 10):
        bad("TASP_ERR_INVALID_ARG", **{f"_{i}": None})
        bad("TASP_ERR_INVALID_ARG", **{f"_{i}": rows(p=FAKE + 8)})
        bad("TASP_ERR_INVALID_ARG", **{f"_{i}": rows(token=1028)})
        bad("TASP_ERR_INVALID_ARG", **{f"_{i}": rows(head=130)})
    bad("TASP_ERR_SHAPE", _9=-1)
    bad("TASP_ERR_SHAPE", _9=513)
    bad("TASP_ERR_INVALID_ARG", _9=0)                  # q with no query heads
    bad("TASP_ERR_SHAPE", _2=rope(rot_dim=136))
    bad("TASP_ERR_INVALID_ARG", _2=rope(theta=1.0))
    bad("TASP_ERR_INVALID_ARG", _2=rope(layout=3))


def test_read_refusals():
    ok = [cache(), 0, None, 4, B.F32, rows(), rows(), None]
    for at, status in (({0: None}, "TASP_ERR_INVALID_ARG"), ({1: 2}, "TASP_ERR_SHAPE"), ({2: FAKE + 1}, "TASP_ERR_INVALID_ARG"), ({3: 0}, "TASP_ERR_SHAPE"),
                       ({3: (1 << 31) - 1}, "TASP_ERR_SHAPE"), ({4: B.E4M3}, "TASP_ERR_INVALID_ARG"), ({5: None}, "TASP_ERR_INVALID_ARG"),
                       ({6: rows(p=FAKE + 4)}, "TASP_ERR_INVALID_ARG")):
        refused(status, B.tasp_page_read, *changed(ok, at))


def test_attention_refusals():
    ok = [cache(), 1, FAKE, 5, B.F32, rows(), 8, 0.1, 100, 3, rows(), FAKE, 1 << 40, None]

    def bad(status, **at):
        refused(status, B.tasp_page_attention, *changed(ok, {int(k[1:]): v for k, v in at.items()}))

    bad("TASP_ERR_INVALID_ARG", _0=None)
    bad("TASP_ERR_SHAPE", _1=2)
    bad("TASP_ERR_SHAPE", _2=None)
    bad("TASP_ERR_INVALID_ARG", _2=FAKE + 1)
    bad("TASP_ERR_SHAPE", _3=0)
    bad("TASP_ERR_SHAPE", _3=B.PAGE_MAX_TOKENS + 1)
    bad("TASP_ERR_INVALID_ARG", _4=9)
    for i in (5, 10):
        bad("TASP_ERR_INVALID_ARG", **{f"_{i}": None})
        bad("TASP_ERR_INVALID_ARG", **{f"_{i}": rows(head=66)})
    for n in (0, 6, 36):
        bad("TASP_ERR_SHAPE", _6=n)
    for s in (0.0, -1.0, float("nan"), float("inf"), 1e300):
        bad("TASP_ERR_INVALID_ARG", _7=s)
    bad("TASP_ERR_SHAPE", _8=-1)
    bad("TASP_ERR_SHAPE", _8=321)
    bad("TASP_ERR_SHAPE", _9=0)
    bad("TASP_ERR_SHAPE", _9=-4)
    long = dict(_0=cache(max_pages=1000), _8=30000)
    bad("TASP_ERR_INVALID_ARG", _11=None, **long)
    bad("TASP_ERR_WORKSPACE", _11=FAKE + 16, **long)
    bad("TASP_ERR_WORKSPACE", _12=64, **long)
    refused("TASP_ERR_SHAPE", B.tasp_page_attention_workspace_bytes, cache(), 6, 5, 100, 5)
    refused("TASP_ERR_SHAPE", B.tasp_page_attention_workspace_bytes, cache(), 8, 5, 1000, 5)
    refused("TASP_ERR_SHAPE", B.tasp_page_attention_workspace_bytes, cache(), 8, 5, 100, 0)
    lib = B.load()
    c = cache()
    assert lib.tasp_page_attention_workspace_bytes(C.addressof(c), 8, 5, 100, 5, None) == -1


def test_attention_workspaces_stay_small():
    """Records of about as many workgroups as the card runs at once, whatever the lengths are."""
    B.load()
    for lens in (0, 1000, 1 << 20):
        for n, new in ((1, 1), (64, 1), (512, 512), (100000, 40000)):
            c = cache(batch=min(n, 256), max_pages=1 << 15, n_kv_heads=8)
            assert B.tasp_page_attention_workspace_bytes(c, 64, n, lens, new) < 400 << 20


def test_logprob_refusals():
    ok = [FAKE, B.F32, 100, FAKE, 5, 100, 1.0, 3, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 2, FAKE, FAKE, 1 << 40, None]

    def bad(status, **at):
        refused(status, B.tasp_token_logprobs, *changed(ok, {int(k[1:]): v for k, v in at.items()}))

    for i in (0, 3, 8, 11, 12):
        bad("TASP_ERR_INVALID_ARG", **{f"_{i}": None})
    for i in (0, 3, 8, 9, 10, 11, 12, 13, 15):
        bad("TASP_ERR_INVALID_ARG", **{f"_{i}": FAKE + 2})
    bad("TASP_ERR_INVALID_ARG", _1=B.BF16, _0=FAKE + 1)
    bad("TASP_ERR_INVALID_ARG", _1=B.INT8)
    bad("TASP_ERR_SHAPE", _2=99)
    for n in (0, -5, 1 << 24):
        bad("TASP_ERR_SHAPE", _4=n)
    for n in (0, (1 << 24) + 1):
        bad("TASP_ERR_SHAPE", _5=n, _2=1 << 40)
    for t in (0.0, -1.0, 1e-31, 1e31, float("nan")):
        bad("TASP_ERR_INVALID_ARG", _6=t)
    bad("TASP_ERR_SHAPE", _7=-1)
    bad("TASP_ERR_SHAPE", _7=33)
    bad("TASP_ERR_INVALID_ARG", _13=None)              # start and mean go together
    bad("TASP_ERR_INVALID_ARG", _15=None)
    bad("TASP_ERR_SHAPE", _14=0)
    bad("TASP_ERR_INVALID_ARG", _5=20000, _2=20000, _16=None)
    bad("TASP_ERR_WORKSPACE", _5=20000, _2=20000, _16=FAKE + 8)
    bad("TASP_ERR_WORKSPACE", _5=20000, _2=20000, _17=10)
    refused("TASP_ERR_SHAPE", B.tasp_token_logprobs_workspace_bytes, 0, 100, 3)
    refused("TASP_ERR_SHAPE", B.tasp_token_logprobs_workspace_bytes, 5, 100, 40)


def test_tensor_wrappers_refuse():
    """Types, shapes and devices that the wrappers check before any address is taken."""
    k = torch.zeros((1, 4, 2, 16, 64), dtype=torch.bfloat16)
    table, ln = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        S.PageCache(k, k, table, ln)
    with pytest.raises(ValueError, match="bfloat16, int8"):
        S.PageCache(k.float(), k.float(), table, ln)
    with pytest.raises(ValueError, match="max_pages"):
        S.PageCache(k, k, table[0], ln)
    with pytest.raises(ValueError, match="GPU"):
        S.token_logprobs(torch.zeros((2, 3)), torch.zeros(2, dtype=torch.int32))
