"""New lengths written over what a commit reads: the lengths themselves, the counts, the path, in place or shifted."""
import pytest
import torch

from paper_2609_29499_amd import session as S
from tests.seq_case import flush

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("over", ["len", "n", "path"])
@pytest.mark.parametrize("shift", [0, 1, -1, 100])
def test_lengths_over_what_the_commit_reads(over, shift):
    """256 sequences, so that four waves hold lengths: as many sums as with an array apart."""
    flush(f"case lengths over {over} shifted {shift}")
    Bn, T, H, S_ = 256, 4, 1, 64
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 40, (Bn,), generator=g).to(torch.int32)
    n = torch.randint(1, T + 1, (Bn,), generator=g).to(torch.int32)
    path = torch.sort(torch.randint(0, T, (Bn, T), generator=g), -1).values.to(torch.int32)
    apart = torch.zeros(Bn, dtype=torch.int32, device="cuda")
    caches = []
    for case in range(2):
        # room on both sides of each array
        bufs = {k: torch.full((128 + v.numel() + 128,), 77, dtype=torch.int32, device="cuda") for k, v in (("len", lens), ("n", n), ("path", path))}
        t = {}
        for k, v in (("len", lens), ("n", n), ("path", path)):
            t[k] = bufs[k][128:128 + v.numel()].view(v.shape)
            t[k].copy_(v)
        k = torch.arange(S_, dtype=torch.float32)[None, None, None, :, None].expand(1, Bn, H, S_, 64).to(torch.bfloat16).contiguous().cuda()
        c = S.SeqCache(k, k.clone(), t["len"])
        out = apart if case == 0 else bufs[over][128 + shift:128 + shift + Bn]
        got = S.seq_commit(c, t["path"], t["n"], len_out=out)
        torch.cuda.synchronize()
        assert got.tolist() == (lens + n).tolist(), case
        caches.append(c)
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)
