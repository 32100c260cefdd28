"""Beam selection where a row's sum is one term and little else: a mask that leaves
one token, probabilities near one.  Scores there are zero or far below one, so that
an error of the sum shows in them, and ties with finished rows hang on it."""
import math

import numpy as np
import pytest

from tests import group_reference as gref
from tests.test_gpu_beam import check, select

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,at", [(1, 0), (1000, 3), (2048, 2047), (151936, 70000), (1 << 19, (1 << 19) - 1)])
@pytest.mark.parametrize("rows", [2, 5])
def test_a_mask_that_leaves_one_token(V, at, rows):
    """Its probability is one and its score the row's, to the bit: a tie with finished rows, which the lower row wins."""
    x = np.full((rows, V), -np.inf, np.float32)
    x[:, at] = np.linspace(-30, 40, rows)
    done = np.arange(rows) % 2
    for s in (0.0, -2.5, -0.1):
        scores = np.full(rows, s, np.float32)
        tok, par, got, fin = select(x, scores, rows, rows, finished=done, end=0)
        assert par.tolist() == [list(range(rows))]
        assert tok.tolist() == [[0 if d else at for d in done]]
        assert (got == scores).all()
        check((tok, par, got, fin), gref.beam_select(x, scores, rows, rows, finished=done, end=0))


@pytest.mark.parametrize("V", [100, 2500, 40001, 151936])
@pytest.mark.parametrize("gap", [20, 30, 33, 36, 60, 800])
def test_a_probability_near_one(V, gap):
    """One logit of 0 and others about gap below: scores of -V e^-gap and less beside a sum of one, which is held to 64
    additions' roundings (a thread's 32, the tree's 12, the parts' 20): 64 half steps of 2^-53."""
    rng = np.random.default_rng(V + gap)
    x = (-gap - rng.random((3, V))).astype(np.float32)
    x[:, V // 3] = 0
    s = np.zeros(3, np.float32)
    tok, par, got, _ = select(x, s, 1, 1)
    for r in range(3):
        want = -math.log1p(math.fsum(np.exp(np.delete(x[r], V // 3).astype(np.float64)).tolist()))
        assert tok[r, 0] == V // 3 and par[r, 0] == r
        assert abs(got[r, 0] - want) <= 2.0**-24 * abs(want) + 64 * 2.0**-53, (r, got[r, 0], want)
