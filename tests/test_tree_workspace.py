"""slim_workspace_bytes_tree in all three sizes that change from step to step.  CPU only."""
import itertools
import random

import pytest

from paper_2503_05840_amd import binding

WIDTHS = [(32, 4096, "bf16"), (20, 1280, "bf16"), (24, 2304, "bf16"), (8, 64, "bf16"), (1, 1024, "bf16"), (130, 1040, "bf16"), (16, 1024, "f32"), (4, 1040, "f32")]


@pytest.mark.parametrize("H,d,dtype", WIDTHS)
def test_a_smaller_batch_tree_or_context_never_needs_more(H, d, dtype):
    size = lambda B, N, T: binding.slim_workspace_bytes_tree(B, N, H, T, d, dtype)      # noqa: E731
    rng = random.Random(H * d)
    batches = [*range(1, 40), 63, 64, 65, 127, 128, 129, 200, 256, 257, 500]
    contexts = [0, 1, 100, 191, 192, 193, 777, 1500, 4096, 16384, 70000]
    for N, T in itertools.product((1, 4, 13, 16, 17, 33, 64), contexts):
        sizes = [size(B, N, T) for B in batches]
        assert sizes == sorted(sizes), (N, T)
    for B, T in itertools.product((1, 2, 5, 16, 33, 128, 200), contexts):
        sizes = [size(B, N, T) for N in range(1, 65)]
        assert sizes == sorted(sizes), (B, T)
    for _ in range(2000):
        B, N, T = rng.randint(1, 300), rng.randint(1, 64), rng.randint(0, 20000)
        assert size(B, N, T) >= size(rng.randint(1, B), rng.randint(1, N), rng.randint(0, T))
