"""Workspaces made with the default arguments serve the calls made with them, with start and without."""
import pytest
import torch

import synth
from paper_2609_29499_amd import session as S
from synth.configs import Shape
from tests.page_case import starts
from tests.seq_case import flush
from tests.test_gpu_page_forward import fill, pool
from tests.test_gpu_tree_step import plan_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hkv,dh,batch,L", [(1, 64, 8, 130), (2, 128, 8, 190), (4, 64, 20, 250), (1, 128, 60, 300)])
def test_default_workspaces(hkv, dh, batch, L):
    flush(f"case workspaces {hkv} {dh} {batch} {L}")
    sh = Shape(1, 512, 8 * hkv, hkv, dh, 512)
    plan = plan_of(sh, None, batch, 64)[-1]
    lens = [L - b for b in range(batch)]
    cache = pool(plan, sh, lens, [1] * batch, 16, "bf16", 3)
    fill(cache, sh, lens, 4)
    x = torch.from_numpy(synth.activations(batch, sh.d_model, 5)).cuda()
    q = torch.randn((batch, 8 * hkv, dh), device="cuda")
    for at in (None, starts([1] * batch).cuda()):
        want = plan.page_forward(x, cache, at)
        got = plan.page_forward(x, cache, at, workspace=plan.page_workspace(cache, batch))
        assert torch.equal(got, want)
        for y in (q, q.bfloat16()):
            ws = S.page_attention_workspace(cache, 8 * hkv, batch)
            assert torch.equal(S.page_attention(cache, 0, y, at, workspace=ws), S.page_attention(cache, 0, y, at))
