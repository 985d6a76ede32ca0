"""A plan's step over drafted tokens with any rotary base that plans take, against the float64 oracle."""
import pytest
import torch

import synth
from oracle import reference as ref
from synth.configs import Shape
from tests.helpers import assert_parity
from tests.seq_case import flush
from tests.test_gpu_tree_step import fill, held, plan_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("theta", [1.0, 0.5, 3.0])
def test_any_rope_base_that_a_plan_takes(theta):
    """Bases down to one and below it, which decode and prefill run too."""
    flush(f"case rope base {theta}")
    sh = Shape(1, 512, 8, 2, 64, 1536, rope_theta=theta)
    lens, T, max_seq = [20, 3], 4, 32
    store, fn, lm, plan = plan_of(sh, None, 2 * T, max_seq)
    cache, caches = fill(plan, sh, "bf16", lens, max_seq, 5)
    x = synth.activations(2 * T, sh.d_model, 3).reshape(2, T, sh.d_model)
    out = plan.tree_forward(torch.from_numpy(x).cuda(), cache)
    torch.cuda.synchronize()
    closed = ref.close_mask(*synth.all_kept_mask(sh), sh.group_size)
    for b in range(2):
        own = [(k[b].copy(), v[b].copy()) for k, v in caches]
        want = ref.prefill_stack(lambda l: store[l], closed, x[b], own, lens[b], sh, fn, lm, kv_store=held("bf16"))
        assert_parity(out[b].double().cpu().numpy(), want, sum_rel=2e-3, what=f"seq {b}")
