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


# (B, N, H, d_k, T, dtype, lens, base, banded): sequence 0's drafted keys lie on both sides of a border of 256 rows, behind whole steps of 64
ACROSS = [
    (2, 20, 4, 64, 250, "bf16", [250, 130], None, False), (2, 20, 4, 64, 250, "f32", [250, 130], None, False),          # one score tile a wave
    (2, 12, 4, 64, 700, "bf16", [505, 700], None, False), (1, 40, 8, 64, 1010, "f32", None, None, False),                # slots shared: the merge
    (2, 9, 6, 72, 1018, "bf16", [1018, 1000], 10000.0, True),
    (3, 20, 72, 16, 1015, "bf16", [1015, 767, 0], None, False), (3, 20, 72, 16, 1015, "bf16", [1015, 767, 0], 500.0, False),      # two score tiles a wave
    (4, 16, 64, 8, 1020, "bf16", [1020, 255, 1000, 0], None, True), (4, 16, 64, 4, 1020, "f32", [1020, 255, 1000, 0], None, False),     # four
    (5, 64, 16, 104, 1785, "bf16", [1785, 1785, 900, 64, 0], None, False),                                               # walks of three blocks, a slot a sequence
    (4, 4, 16, 52, 2302, "f32", [2302, 2303, 1500, 9], None, False), (1, 26, 8, 128, 16375, "bf16", None, None, False),  # walks, slots shared
]


@pytest.mark.parametrize("i", range(len(ACROSS)))
def test_drafted_keys_across_a_row_block(i):
    B, N, H, d_k, T, dtype, lens, base, banded = ACROSS[i]
    say(f"[case] tree, odd key about a border: B={B} N={N} H={H} d_k={d_k} T={T} {dtype} base={base} banded={banded}")
    n = T if lens is None else lens[0]
    left = 256 - n % 256
    assert 0 < left < N and n >= 64
    for node, value in ((left - 1, np.nan), (left, np.inf), (left, np.nan), (N - 1, -np.inf)):
        c = TreeCase(B, N, H, d_k, T, dtype, lens=lens, base=base, banded=banded, seed=700 + i, slack=40)
        check_odd_keys(c, node, [c.d - 2], value)
