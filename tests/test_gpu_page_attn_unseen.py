"""What a token does not see reaches nothing: finite values of any size in later rows and pages. Tolerances: those of test_gpu_page_attn.check."""
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
