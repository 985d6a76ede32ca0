"""What a call's shape says about its workspace (host only): long sequences are cut into chunks, whatever number of others there is."""
import pytest

from paper_2609_29499_amd import binding as B
from tests.test_page_cpu import cache


@pytest.mark.parametrize("heads,hq", [(8, 32), (8, 64), (2, 8)])
@pytest.mark.parametrize("batch,n,new", [(1, 1, 1), (32, 32, 1), (64, 64, 1), (256, 256, 1), (60, 300, 5), (4, 8195, 8192)])
def test_long_sequences_are_cut(heads, hq, batch, n, new):
    B.load()
    c = cache(batch=batch, max_pages=4096, n_kv_heads=heads)
    long = B.tasp_page_attention_workspace_bytes(c, hq, n, 131072, new)
    assert 0 < long < 100 << 20
    assert B.tasp_page_attention_workspace_bytes(c, hq, n, 100, min(new, 4)) == 0          # no step that could be cut
