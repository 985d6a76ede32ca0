"""What a token does not see reaches nothing: finite values of any size in later rows and pages, scales that the values seen do not
reach, queries of tokens without rows. Tolerances: those of test_gpu_page_attn.check."""
import math

import pytest
import torch

from paper_2609_29499_amd import session as S
from tests.page_case import paged, starts
from tests.seq_case import DTYPES, flush, randn
from tests.test_gpu_page_attn import check, edges

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("lens,n,hq,dh,P", [([0, 40], [70, 70], 8, 64, 16), ([0], [200], 4, 128, 32), ([33, 0], [150, 64], 8, 128, 16),
                                            ([4001, 7], [100, 90], 7, 128, 32), ([130, 9], [3, 2], 4, 64, 16)])
def test_large_values_of_later_tokens(kind, act, lens, n, hq, dh, P):
    """The values of a later token's row (8 bits: of a page that holds later tokens only) are 2^60 times as large: tokens that do
    not see it keep their bits, and the others have what the oracle says."""
    flush(f"case later values {kind} {act} {lens} {n} {hq} {dh} {P}")
    c, rows = paged(lens, n, 1, P, dh, kind, 71)
    q = randn((sum(n), hq, dh), DTYPES[act], 72)
    at = starts(n).cuda()
    clean = S.page_attention(c, 0, q.cuda(), at)
    torch.cuda.synchronize()
    check(clean.double().cpu().numpy(), q.double().numpy(), rows[0], lens, n, P, act, dh ** -0.5, some=edges)
    kept, t = [], 0
    for b, (L, m) in enumerate(zip(lens, n)):
        r = L + m - 1 if kind == "bf16" else (L + m - 1) // P * P      # the first row that is changed
        page = int(c.table[b, r // P])
        if kind == "bf16":
            c.v[0, page, :, r % P] *= 2.0 ** 60
            rows[0][b][1][r] *= 2.0 ** 60
        else:
            c.v_scale[0, page] *= 2.0 ** 60
            rows[0][b][1][r:r + P] *= 2.0 ** 60
        kept += range(t, t + max(0, r - L))
        t += m
    got = S.page_attention(c, 0, q.cuda(), at)
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, n, P, act, dh ** -0.5, some=edges)
    assert torch.equal(got[kept], clean[kept])


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("power", [3, 5, 40])
@pytest.mark.parametrize("lens,n,hq,dh,P", [([700, 5], [40, 40], 8, 128, 128), ([300], [600], 1, 128, 64), ([900, 300], [20, 33], 8, 64, 16)])
def test_scales_above_the_values_seen(kind, power, lens, n, hq, dh, P):
    """A page's scale goes by all that was written into it: here the rows that are left hold nothing but zeros, at the front or
    in the middle, under scales of up to 2^40 times the others'."""
    flush(f"case scales above {kind} {power} {lens} {n} {hq} {dh} {P}")
    for j in (0, 1):
        c, rows = paged(lens, n, 1, P, dh, kind, 73)
        for b in range(len(lens)):
            j_ = min(j, lens[b] // P)
            page = int(c.table[b, j_])
            c.v.view(torch.uint8 if kind == "e4m3" else torch.int8)[0, page] = 0
            c.v_scale[0, page] = c.v_scale.max() * 2.0 ** power
            rows[0][b][1][j_ * P:(j_ + 1) * P] = 0.0
        q = randn((sum(n), hq, dh), torch.bfloat16, 74)
        got = S.page_attention(c, 0, q.cuda(), starts(n).cuda())
        torch.cuda.synchronize()
        check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, n, P, "bf16", dh ** -0.5, some=edges)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("L,n,hq,what", [(3000, 20, 4, math.inf), (3000, 9, 2, -math.inf), (40, 30, 8, math.inf), (3005, 400, 4, math.nan)])
def test_queries_of_absent_tokens(L, n, hq, what, kind, act):
    """Tokens beyond the table's pages, in one chunk and in several, whose queries are not finite: zeros, and the others as they were."""
    flush(f"case absent {L} {n} {hq} {what} {kind} {act}")
    P, dh = 16, 64
    c, rows = paged([L], [8], 1, P, dh, kind, 75)
    q = randn((n, hq, dh), DTYPES[act], 76)
    absent = c.max_seq - L
    assert 0 < absent < n
    clean = S.page_attention(c, 0, q.cuda(), starts([n]).cuda())
    q[absent:, :, 0] = what             # (scores of one sign: the running maximum is infinite too)
    got = S.page_attention(c, 0, q.cuda(), starts([n]).cuda())
    torch.cuda.synchronize()
    assert not got[absent:].any() and torch.equal(got[:absent], clean[:absent])


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("n", [1, 3, 40])
@pytest.mark.parametrize("what", [math.inf, math.nan])
def test_queries_that_see_no_row(what, n, kind, act):
    """Sequences without any page (places of a step that no conversation has), whose queries hold anything: zeros."""
    flush(f"case no row {what} {n} {kind} {act}")
    P, dh, hq = 16, 64, 8
    lens = [0, 50, 2500, 3000]
    c, _ = paged(lens, [n] * 4, 1, P, dh, kind, 77)
    q = randn((4 * n, hq, dh), DTYPES[act], 78)
    at = None if n == 1 else starts([n] * 4).cuda()
    clean = S.page_attention(c, 0, q.cuda(), at).view(4, n, hq, dh)
    c.table[0] = -1
    c.table[2] = c.n_pages
    q.view(4, n, hq, dh)[::2, :, :, 1::2] = what
    got = S.page_attention(c, 0, q.cuda(), at).view(4, n, hq, dh)
    torch.cuda.synchronize()
    assert not got[::2].any() and torch.equal(got[1::2], clean[1::2])
