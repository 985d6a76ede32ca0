"""Limits of the drafted-token entry points that are checked before any GPU work."""
import pytest
import torch

from paper_2609_29499_amd import binding as B
from paper_2609_29499_amd import session as S
from tests.test_seq_cpu import FAKE, cache, refused, rope, rows


@pytest.mark.parametrize("dh,n", [(128, ((1 << 24) - 1) * 16 + 1), (64, ((1 << 24) - 1) * 32 + 1), (128, 2 ** 31 - 1), (64, 2 ** 31 - 1)])
def test_reads_of_more_rows_than_a_launch_has(dh, n):
    """A workgroup reads 2048 / dh rows, and a launch has fewer than 2^24 of them in a dimension."""
    refused("TASP_ERR_SHAPE", B.tasp_seq_read, cache(head_dim=dh), 0, None, n, B.BF16, rows(), rows(), None)


def test_a_cache_keeps_the_tensors_that_it_names():
    """Another tensor under a cache's name would leave the library with the address of one that torch frees."""
    c = S.SeqCache.__new__(S.SeqCache)
    for name in ("k", "v", "len", "k_scale", "v_scale", "struct", "max_seq", "batch"):
        setattr(c, name, torch.zeros(3))
        with pytest.raises(AttributeError, match=name):
            setattr(c, name, torch.ones(3))
        assert not getattr(c, name).any()
    kept = c.len
    c.len += 1                                         # (in place)
    assert c.len is kept and c.len.tolist() == [1, 1, 1]


def test_workspaces_of_another_device():
    ws = S._workspace(512, "cpu")
    with pytest.raises(ValueError, match="workspace"):
        S._on(0, ws)
    assert S._on(-1, ws) is ws and S._on(0, (None, 256, 16)) == (None, 256, 16)


def test_numbers_that_leave_their_types():
    """A scale that is infinite in 32 bits, a factor whose reciprocal is infinite in 64."""
    c = cache(batch=1)
    for s in (1e300, 3e38, 2.0 ** 128):
        refused("TASP_ERR_INVALID_ARG", B.tasp_tree_attention, c, 0, None, 1, B.BF16, rows(), 8, s, 100, rows(), FAKE, 1 << 40, None)
    for scaling in (1, 2, 3):
        refused("TASP_ERR_INVALID_ARG", B.tasp_seq_append, c, 0, rope(scaling=scaling, factor=1e-310), None, 1, B.BF16, None,
                rows(), rows(), 0, None, None)
