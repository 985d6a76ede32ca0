"""Pins of the token score oracle: torch's log_softmax, closed forms, ties, padding and rows without logits."""
import math

import numpy as np
import torch

from oracle import score as O


def test_against_log_softmax_and_topk():
    x = np.random.default_rng(0).standard_normal(300) * 3
    for temperature in (0.5, 1.0, 2.0):
        lp = torch.log_softmax(torch.tensor(x) / temperature, -1)
        got = O.score(x, 17, temperature, 8)
        assert math.isclose(got[0], float(lp[17]), rel_tol=1e-12)
        assert math.isclose(got[1], float(-(lp.exp() * lp).sum()), rel_tol=1e-12)
        top = torch.topk(lp, 8)
        assert got[3] == top.indices.tolist() and np.allclose(got[4], top.values, rtol=1e-12)
        assert got[2] == int((x > x[17]).sum())


def test_closed_forms():
    lp, h, rank, ids, tops = O.score([2.0] * 8, 5, 1.0, 3)
    assert math.isclose(lp, -math.log(8)) and math.isclose(h, math.log(8)) and rank == 5 and ids == [0, 1, 2]
    lp, h, rank, ids, tops = O.score([0.0, math.log(3.0)], 0, 1.0, 2)
    assert math.isclose(lp, -math.log(4)) and ids == [1, 0] and rank == 1
    assert math.isclose(h, 0.25 * math.log(4) + 0.75 * math.log(4 / 3))


def test_borders():
    inf, nan = math.inf, math.nan
    assert O.score([-inf, nan, -inf], 1, 1.0, 2) == (-inf, 0.0, 1, [-1, -1], [-inf, -inf])
    lp, h, rank, ids, tops = O.score([1.0, inf, -inf, inf], 3, 1.0, 4)
    assert math.isclose(lp, -math.log(2)) and math.isclose(h, math.log(2)) and rank == 1 and ids == [1, 3, 0, -1]
    assert tops[2:] == [-inf, -inf]
    assert O.score([1.0, 2.0], -1)[::2][:2] == (0.0, -1) and O.score([1.0, 2.0], 2)[2] == -1
    assert O.mean([-1.0, -2.0, 0.0, -4.0], [0, 1, -1, 1], 2, [0, 3, 3, 9]) == [-1.5, 0.0, -4.0]
