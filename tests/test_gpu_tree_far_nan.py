"""slim_tree_decode with a row of context that is not finite where a head gives it a weight too small for fp32: the result is NaN, however the rows are cut."""
import numpy as np
import pytest

from paper_2503_05840_amd import synth
from gpu_harness import say
from tree_cases import TreeCase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [1, 130])
@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_a_row_of_vanishing_weight(B, dtype, value):
    say(f"[case] tree, context {value} without weight: B={B} {dtype}")
    c = TreeCase(B, 3, 2, 32, 1500, dtype, parents=[[-1, 0, 7]] * B, seed=51)      # (slot 2 is unused)
    c.q[:] = synth.round_through(np.abs(c.q) + 1.0, dtype)
    c.K[:, :700, :32] = -100.0                                   # head 0: scores far below those of the other rows
    clean = c.run()
    assert np.isfinite(clean).all()
    c.K[:, 5, 40] = value                                        # a column of head 1, whose score of this row is not finite either
    got = c.run()
    assert not np.isfinite(got[:, :2]).any()
    assert (got[:, 2] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[0], None])
def test_a_key_whose_score_is_minus_infinity(dtype, lens):
    """No numerator is left for a node whose only key has a score of minus infinity; it is NaN all the same, unlike an unused slot."""
    say(f"[case] tree, score of minus infinity: {dtype} lens={lens}")
    c = TreeCase(1, 3, 2, 32, 1500 if lens else 0, dtype, lens=lens, parents=[[-1, 0, 7]], seed=52)
    c.q[:] = synth.round_through(np.abs(c.q) + 1.0, dtype)
    c.K[0, 0, :] = -np.inf
    got = c.run()
    assert not np.isfinite(got[:, :2]).any() and (got[:, 2] == 0).all()
