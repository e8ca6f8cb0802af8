"""The example's speculative steps give the tokens of one step after the other."""
import os
import sys

import pytest

from gpu_harness import say

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_speculative_steps_are_lossless():
    import speculative_step as ex
    say("[case] example: speculative steps against single ones")
    model = ex.Model(V=128, H=4, d=128)
    keys, lens, last = ex.prompts(model, B=3, T=120)
    got = ex.speculative(model, keys, lens, last, steps=16)
    want = ex.one_by_one(model, keys, lens, last, max(len(t) for t in got))
    for mine, ref in zip(got, want):
        assert len(mine) >= 16 and mine == ref[:len(mine)]
    assert sum(len(t) for t in got) > 3 * 16          # (some drafted tokens were accepted)
