"""Limits of the drafted-token entry points that are checked before any GPU work."""
import pytest

from paper_2609_29499_amd import binding as B
from tests.test_seq_cpu import cache, refused, rows


@pytest.mark.parametrize("dh,n", [(128, ((1 << 24) - 1) * 16 + 1), (64, ((1 << 24) - 1) * 32 + 1), (128, 2 ** 31 - 1), (64, 2 ** 31 - 1)])
def test_reads_of_more_rows_than_a_launch_has(dh, n):
    """A workgroup reads 2048 / dh rows, and a launch has fewer than 2^24 of them in a dimension."""
    refused("TASP_ERR_SHAPE", B.tasp_seq_read, cache(head_dim=dh), 0, None, n, B.BF16, rows(), rows(), None)
