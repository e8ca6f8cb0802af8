"""slim_tree_decode where workgroups of the scores walk over several blocks of 256 rows: one to four query tiles a head, both types, one sequence
and ragged batches, with references of the softmax numerators that differ by many steps from one block to the next, so that a block
that got its neighbour's reference would have its weight off by a large power of two."""
import numpy as np
import pytest

from paper_2503_05840_amd import synth
from gpu_harness import say
from tree_cases import TreeCase

pytestmark = pytest.mark.gpu

# (B, N, H, d_k, T, dtype, lens, sequences looked at, nodes looked at).  All have more than 512 (head, block, sequence) workgroups, at most 256 (head, sequence) pairs
# and heads of 97 to 128 columns (fp32: 49 to 64): three blocks or more to a workgroup, the last one's ends in the drafted rows.
WALKS = [
    (8, 16, 4, 104, 4300, "bf16", [4300, 4097, 4096, 4080, 2500, 700, 0, 3000], [0, 2, 3, 6], [0, 7, 15]),         # one tile, slots shared
    (22, 34, 8, 128, 734, "bf16", [734 - 31 * i for i in range(22)], [0, 4, 20], [0, 13, 33]),                     # three tiles, a slot a sequence
    (5, 64, 16, 104, 1900, "bf16", [1900, 1792, 1785, 1000, 40], [0, 2, 4], [0, 31, 63]),                          # four tiles, a slot a sequence, 30 steps
    (1, 26, 8, 128, 16390, "bf16", None, [0], [0, 25]),                                                            # three tiles, one sequence in many slots
    (17, 64, 8, 64, 950, "f32", [950 - 55 * i for i in range(17)], [0, 3, 16], [0, 30, 63]),                       # four tiles, a slot a sequence
    (4, 4, 16, 52, 2310, "f32", [2310, 2304, 1500, 9], [0, 1, 3], [0, 3]),                                         # one tile, slots shared
]


@pytest.mark.parametrize("i", range(len(WALKS)))
@pytest.mark.parametrize("far", [False, True])
def test_walk_over_row_blocks(i, far):
    B, N, H, d_k, T, dtype, lens, sequences, nodes = WALKS[i]
    say(f"[case] tree, walk: B={B} N={N} H={H} d_k={d_k} T={T} {dtype} far={far}")
    assert H * B * ((T + N + 255) // 256) > 512 and H * B <= 256
    c = TreeCase(B, N, H, d_k, T, dtype, lens=lens, seed=500 + i, q_scale=40.0 if far else 1.5)
    if far:
        # maxima of the blocks' scores (log2): about 170, 4, 50, 170, ...
        scale = np.array([1.0, 0.02, 0.3])[np.arange(c.rows) // 256 % 3]
        c.K = synth.round_through(c.K * scale[None, :, None], dtype)
    say(f"       {c.check_some(sequences, nodes):.3f} of the bound")


@pytest.mark.parametrize("dtype,d_k", [("bf16", 8), ("f32", 4)])
@pytest.mark.parametrize("N", [3, 6, 9, 12, 17, 24])
@pytest.mark.parametrize("far", [False, True])
def test_a_slot_a_sequence_over_many_steps(N, dtype, d_k, far):
    """More sequences than half the compute units: none is cut, whatever its length.  One to eight query tiles a wave, up to 15 steps of 64 rows."""
    B, H, T = 130, 5, 900
    say(f"[case] tree, a slot a sequence: B={B} N={N} H={H} d_k={d_k} T={T} {dtype} far={far}")
    c = TreeCase(B, N, H, d_k, T, dtype, lens=[(901 - 53 * i) % 901 for i in range(B)], seed=600 + N, q_scale=40.0 if far else 1.5)
    if far:
        scale = np.array([0.02, 1.0, 0.3, 1.0])[np.arange(c.rows) // 256 % 4]
        c.K = synth.round_through(c.K * scale[None, :, None], dtype)
    say(f"       {c.check_some([0, 1, 2, 16, 17, 77, 129], [0, N // 2, N - 1]):.3f} of the bound")
