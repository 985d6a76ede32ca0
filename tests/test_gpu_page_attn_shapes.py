"""Steps whose sequences differ in their lengths and numbers of new tokens by far, over the rules that choose kernels, blocks and
chunks from a call's shape. Tolerances: those of test_gpu_page_attn.check."""
import pytest
import torch

from paper_2609_29499_amd import session as S
from tests.page_case import paged, starts
from tests.seq_case import DTYPES, flush, randn
from tests.test_gpu_page_attn import check

pytestmark = pytest.mark.gpu


def attended(lens, n, hq, H, dh, P, kind, act, room, max_new=None, **hints):
    """A step against the oracle; the same bits again. room: pages of the tables behind what is needed."""
    c, rows = paged(lens, n, H, P, dh, kind, 81, room=room, spare=0)
    q = randn((sum(n), hq, dh), DTYPES[act], 82)
    at = None if set(n) == {1} and max_new is None else starts(n).cuda()
    got = S.page_attention(c, 0, q.cuda(), at, max_new=max_new, **hints)
    again = S.page_attention(c, 0, q.cuda(), at, max_new=max_new, **hints)
    torch.cuda.synchronize()
    assert torch.equal(got, again)
    check(got.double().cpu().numpy(), q.double().numpy(), rows[0], lens, n, P, act, dh ** -0.5, some=lambda m: [0, 1, 31, 32, m // 2, m - 2, m - 1])


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("lens,n,hq", [([0], [64], 8), ([33, 0], [150, 64], 8), ([5, 0, 9], [513, 1, 2], 1), ([2300, 3, 90], [100, 20, 9], 8),
                                       ([2500], [257], 2), ([100, 0, 64, 31], [70, 65, 130, 1], 8)])
def test_many_query_rows_under_wide_tables(kind, lens, n, hq):
    """512 query rows and more of a sequence where 2048 rows and more may be seen: whole and partial blocks, beside others that
    fill a block, fill little of one, or are single tokens."""
    flush(f"case wide tables {kind} {lens} {n} {hq}")
    attended(lens, n, hq, 1, 128, 32, kind, "bf16", 70)


@pytest.mark.parametrize("kind,dh", [("int8", 128), ("bf16", 64), ("e4m3", 128)])
@pytest.mark.parametrize("lens,n,H", [([1100, 900], [130, 1], 8), ([3000, 2000, 5], [64, 1, 1], 2), ([1500, 10], [300, 3], 16), ([100, 700], [257, 1], 12)])
def test_float32_beside_short_sequences(kind, dh, lens, n, H):
    """One kernel for all, or both: many query rows of one sequence, few of the others, behind short and long rows."""
    flush(f"case float32 {kind} {dh} {lens} {n} {H}")
    attended(lens, n, H, H, dh, 64, kind, "f32", 1, max_new=max(n), max_len=max(lens))
    attended(lens, n, 4, 1, dh, 64, kind, "f32", 1, max_new=max(n), max_len=max(lens))


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kind,dh,hq,H,lens,n", [
    ("int8", 64, 8, 8, [30000] + [100] * 63, [1] * 64), ("bf16", 128, 8, 2, [60] * 200 + [20000] + [0, 1] * 27, [1] * 255),
    ("e4m3", 64, 4, 4, [9000] + [50] * 70, [2, 1, 3] * 23 + [1, 1]), ("int8", 128, 16, 8, [5000 - 61 * b for b in range(80)], [1] * 80),
    ("bf16", 64, 64, 8, [0, 9000, 7000], [2500, 1, 2]), ("e4m3", 128, 16, 2, [10, 20000, 300, 40], [700, 1, 1, 1])])
def test_one_sequence_far_longer_than_the_others(kind, dh, hq, H, lens, n, act):
    """More blocks of query rows than there are workgroups for, and more tokens in a step than single ones: the long sequence is cut."""
    flush(f"case long among short {kind} {dh} {hq} {H} {len(lens)} {max(lens)} {act}")
    attended(lens, n, hq, H, dh, 64, kind, act, 0, max_new=max(n), max_len=max(lens))
