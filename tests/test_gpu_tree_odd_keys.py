"""slim_tree_decode with drafted keys that are not finite: the nodes that see one are NaN, the others keep their bits, wherever the key lies."""
import numpy as np
import pytest

from gpu_harness import say
from tree_cases import TreeCase

pytestmark = pytest.mark.gpu


def check_odd_keys(c, node, columns, value=np.nan, lens=None):
    """Sequence 0's drafted key `node` gets `value` in the columns; every slot behind the drafted ones too."""
    clean = c.run()
    assert np.isfinite(clean).all()
    c.K[0, int(c.lens[0]) + node, columns] = value
    for b in range(c.B):
        c.K[b, int(c.lens[b]) + c.N:] = value
    got = c.run()
    sees = np.zeros((c.B, c.N), dtype=bool)
    for i in range(c.N):
        at = i
        while at >= 0:
            sees[0, i] |= at == node
            at = int(c.parents[0, at])
    assert sees.any()
    assert not np.isfinite(got[sees]).any()
    assert np.array_equal(got[~sees], clean[~sees])


@pytest.mark.parametrize("dtype,vec", [("bf16", 8), ("f32", 4)])
@pytest.mark.parametrize("N,H", [(1, 5), (16, 2), (23, 2), (16, 4), (32, 3), (64, 2)])
def test_contexts_shorter_than_a_step(N, H, dtype, vec):
    """No whole step of 64 rows before the drafted keys: the weighted sum takes all its rows one chunk after the other.  One to eight query tiles a wave."""
    say(f"[case] tree, odd key behind a short context: N={N} H={H} {dtype}")
    for lens in ([0, 63], [17, 40], [63, 0]):
        c = TreeCase(2, N, H, 4 * vec, 63, dtype, lens=lens, seed=31 + N, slack=5)
        check_odd_keys(c, N // 2, [3])
