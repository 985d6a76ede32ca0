"""Packed tokens at the ends of their ranges: as many sequences as a call takes, values near both ends of float32, probabilities
far below the largest, few rows. Tolerances: those of test_gpu_page_attn.check."""
import math

import numpy as np
import pytest
import torch

from paper_2609_29499_amd import session as S
from tests.page_case import paged, starts
from tests.seq_case import DTYPES, flush, gen, randn
from tests.test_gpu_page_attn import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,act", [("int8", "bf16"), ("bf16", "f32")])
def test_as_many_sequences_as_there_may_be(kind, act):
    """256 sequences, most with a token or none, some with many: appended and attended."""
    flush(f"case 256 {kind} {act}")
    g = gen(1)
    n = torch.randint(0, 3, (256,), generator=g).tolist()
    n[0], n[77], n[255] = 50, 1, 41
    lens = torch.randint(0, 90, (256,), generator=g).tolist()
    lens[3], lens[200] = 2000, 0
    H, hq, dh, P = 2, 6, 64, 16
    c, rows = paged(lens, n, H, P, dh, kind, 2)
    N = sum(n)
    at = starts(n).cuda()
    q = randn((N, hq, dh), DTYPES[act], 3)
    # (attended first: the rows of the new tokens are the pool's own)
    got = S.page_attention(c, 0, q.cuda(), at)
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, n, P, act, dh ** -0.5, some=lambda c: [0, c // 2, c - 1])
    k, v = (randn((N, H, dh), DTYPES[act], 4 + i).cuda() for i in range(2))
    S.page_append(c, 0, None, k, v, at)
    S.page_advance(c, N, at)
    assert c.len.tolist() == [a + b for a, b in zip(lens, n)]
    first = torch.tensor(lens, dtype=torch.int32, device="cuda")
    back = S.page_read(c, 0, max(n), first, dtype=torch.float32)
    torch.cuda.synchronize()
    t = 0
    for b, m in enumerate(n):
        for x, y, sc in ((k, back[0], c.k_scale), (v, back[1], c.v_scale)):
            want, have = x[t:t + m].float().transpose(0, 1), y[b, :, :m]
            if kind == "bf16":
                assert torch.equal(have, want.to(torch.bfloat16).float()), b
            else:                       # half a code of the row's page, and the quotient's 2^-22
                page = c.table[b, torch.arange(lens[b], lens[b] + m, device="cuda") // P].long()
                s = sc[0][page].T[:, :, None]
                assert torch.all((have - want).abs() <= s / 2 * (1 + 2.0 ** -20) + want.abs() * 2.0 ** -21), b
        t += m


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("power", [-90, 104])
@pytest.mark.parametrize("dh,n", [(64, 1), (64, 30), (128, 30)])
def test_values_near_both_ends(kind, act, power, dh, n):
    """v times 2^-90 (three terms of a probability times an 8-bit scale stay above 2^-126) and times 2^104 (60 rows of at most 2^9
    stay below 2^120)."""
    flush(f"case ends {kind} {act} {power} {dh} {n}")
    lens, hq, P = [30, 0], 8, 16
    c, rows = paged(lens, [n, n], 1, P, dh, kind, 5)
    assert max(np.abs(r[1]).max() for r in rows[0]) < 2.0 ** 9
    f = 2.0 ** power
    if kind == "bf16":
        c.v.copy_((c.v.double() * f).to(torch.bfloat16))
    else:
        c.v_scale.mul_(f)
    for r in rows[0]:
        r[1][:] = r[1] * f
    q = randn((2 * n, hq, dh), DTYPES[act], 6)
    got = S.page_attention(c, 0, q.cuda(), starts([n, n]).cuda())
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, [n, n], P, act, dh ** -0.5)


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 6, 20])
@pytest.mark.parametrize("last", [False, True])
def test_large_values_under_small_probabilities(kind, act, n, last):
    """The first or the last page's rows score 2^-20 of the others, and their values are 2^24 times as large: both count. Rows that score
    2^-60 and hold as much as the largest count for nothing more."""
    flush(f"case small probabilities {kind} {act} {n} {last}")
    P, dh, hq = 16, 64, 8
    L = 6 * P
    c, rows = paged([L], [n], 1, P, dh, kind, 7, spare=0)
    J = c.table.shape[1]
    power = torch.zeros(J)
    power[J - 1 if last else 0] = -20
    power[2] = -60
    big = torch.ones(J)
    big[J - 1 if last else 0] = 2.0 ** 24
    big[2] = 2.0 ** 24
    for j in range(J):
        page = int(c.table[0, j])
        k = torch.zeros((P, dh))
        k[:, 0] = power[j] / 4          # (small whole numbers: exact in every type)
        c.k[0, page, 0] = k.to(c.k.dtype).cuda()
        if kind == "bf16":
            c.v[0, page] *= big[j].item()
        else:
            c.k_scale[0, page] = 1.0
            c.v_scale[0, page] *= big[j].item()
        rows[0][0][0][j * P:(j + 1) * P, 0] = k.double().numpy()
        rows[0][0][1][j * P:(j + 1) * P] *= big[j].item()
    q = torch.zeros((n, hq, dh), dtype=DTYPES[act])
    q[..., 0] = 4.0
    got = S.page_attention(c, 0, q.cuda(), starts([n]).cuda(), scale=math.log(2.0))
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], [L], [n], P, act, math.log(2.0))


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("lens,n,hq,P", [([33, 0], [150, 64], 8, 16), ([2000, 700, 5], [130, 3, 65], 8, 64), ([0], [513], 1, 128), ([4001], [100], 7, 32)])
def test_large_blocks_of_query_rows(kind, lens, n, hq, P):
    """Heads of 128 with 512 query rows and more of a sequence: whole and partial blocks of 256, in one chunk and in several. Values
    that grow along the cache by 20 powers of two; then NaN and infinities in the last tokens' rows, which earlier ones do not see."""
    flush(f"case large blocks {kind} {lens} {n} {hq} {P}")
    c, rows = paged(lens, n, 1, P, 128, kind, 33)
    J = c.table.shape[1]
    f = torch.exp2(torch.linspace(-10, 10, J).round())
    for b in range(len(lens)):
        for j in range(J):
            page = int(c.table[b, j])
            if page < 0:
                continue
            if kind == "bf16":
                c.v[0, page] *= f[j].item()
            else:
                c.v_scale[0, page] *= f[j].item()
            rows[0][b][1][j * P:(j + 1) * P] *= f[j].item()
    q = randn((sum(n), hq, 128), torch.bfloat16, 34)
    at = starts(n).cuda()
    got = S.page_attention(c, 0, q.cuda(), at)
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, n, P, "bf16", 128 ** -0.5,
          some=lambda m: [0, 1, 31, 32, 63, 64, m // 2, m - 2, m - 1])
    if kind == "int8":
        return
    t = 0
    seen = []
    for b, (L, m) in enumerate(zip(lens, n)):
        r = L + m - 1                   # the last token's own row
        page = int(c.table[b, r // P])
        if kind == "bf16":
            c.v[0, page, :, r % P, ::5], c.v[0, page, :, r % P, 1::5] = math.nan, math.inf
        else:
            c.v.view(torch.uint8)[0, page, :, r % P] = 0x7f
        seen.append(torch.arange(t, t + m - 1))
        t += m
    seen = torch.cat(seen)
    odd = S.page_attention(c, 0, q.cuda(), at)
    torch.cuda.synchronize()
    assert torch.equal(odd[seen], got[seen])
    last = torch.tensor(n).cumsum(0) - 1
    assert not torch.isfinite(odd[last][..., ::5]).any()


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("n,hq,dh", [(40, 8, 64), (40, 8, 128), (64, 1, 64), (9, 8, 128)])
def test_few_rows_keep_the_bits_of_the_probabilities(kind, n, hq, dh):
    """Sums that are often far smaller than their terms: the bound goes by the terms."""
    flush(f"case bits {kind} {n} {hq} {dh}")
    lens = [0, 3, 9]
    c, rows = paged(lens, [n] * 3, 1, 32, dh, kind, 60 + n)
    q = randn((3 * n, hq, dh), torch.bfloat16, 61)
    got = S.page_attention(c, 0, q.cuda(), starts([n] * 3).cuda())
    torch.cuda.synchronize()
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, [n] * 3, 32, "bf16", dh ** -0.5)


def test_what_tokens_of_no_sequence_hold_reaches_nothing():
    """NaN in front of the first and behind the last sequence's rows, 1 and many tokens: nothing of it is written anywhere."""
    for n in ([1, 1], [40, 1500]):
        flush(f"case no sequence {n}")
        H, hq, dh, P, front, behind = 1, 4, 64, 64, 3, 5
        c, _ = paged([10, 0], n, H, P, dh, "int8", 9)
        d, _ = paged([10, 0], n, H, P, dh, "int8", 9)
        N = sum(n)
        q, k, v = (randn((N, h, dh), torch.bfloat16, 10 + i).cuda() for i, h in enumerate((hq, H, H)))
        pad = lambda x: torch.cat([torch.full_like(x[:1], math.nan).expand(front, -1, -1), x,          # noqa: E731
                                   torch.full_like(x[:1], math.nan).expand(behind, -1, -1)])
        rope = S.Rope("half", dh)
        want = S.page_append(c, 0, q, k, v, starts(n).cuda(), rope)
        out = torch.full((N + front + behind, hq, dh), 7.0, dtype=torch.bfloat16, device="cuda")
        S.page_append(d, 0, pad(q), pad(k), pad(v), starts(n, front).cuda(), rope, q_out=out)
        torch.cuda.synchronize()
        assert torch.equal(out[front:front + N], want) and out[:front].eq(7).all() and out[front + N:].eq(7).all()
        for t in ("k", "v", "k_scale", "v_scale"):
            assert torch.equal(getattr(c, t), getattr(d, t)), t


def test_queries_and_their_outputs_in_one_buffer():
    """q and q_out as different heads of the same rows."""
    flush("case one buffer")
    n, H, hq, dh, P = [5, 1100], 2, 4, 64, 16
    c, _ = paged([3, 9], n, H, P, dh, "bf16", 11)
    buf = randn((sum(n), 2 * hq, dh), torch.float32, 12).cuda()
    k, v = (randn((sum(n), H, dh), torch.float32, 13 + i).cuda() for i in range(2))
    rope = S.Rope("half", dh)
    want = S.page_append(c, 0, buf[:, :hq].contiguous(), k, v, starts(n).cuda(), rope)
    S.page_append(c, 0, buf[:, :hq], k, v, starts(n).cuda(), rope, q_out=buf[:, hq:])
    torch.cuda.synchronize()
    assert torch.equal(buf[:, hq:], want)
