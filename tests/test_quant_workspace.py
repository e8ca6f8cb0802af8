"""slim_workspace_bytes_quant in batch and context.  CPU only."""
import random

import pytest

from launch_rules import quant_cut
from paper_2503_05840_amd import binding

WIDTHS = [(32, 4096, "bf16"), (24, 2304, "bf16"), (20, 1280, "f32"), (20, 1280, "bf16"), (16, 1024, "f32"), (1, 32, "bf16"), (1, 512, "f32"), (130, 4160, "bf16"),
          (12, 864, "f32"), (40, 1280, "bf16")]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("H,d,dtype", WIDTHS)
def test_a_smaller_batch_or_context_never_needs_more(H, d, dtype, bits):
    size = lambda B, T: binding.slim_workspace_bytes_quant(B, H, T, d, bits, dtype)      # noqa: E731
    batches = [*range(1, 140), 200, 255, 256, 257, 300, 500, 1000, 1024, 1025, 4095, 4096, 4097, 5000]
    contexts = sorted({1, 63, 64, 65, 128, 129, 777, 1500, 3000, 4096, 5000, 16384, 70000} | set(range(100, 9000, 331)))
    for T in contexts:
        sizes = [size(B, T) for B in batches]
        assert sizes == sorted(sizes) and sizes[0] > 0, T
    for B in batches[::3]:
        sizes = [size(B, T) for T in contexts]
        assert sizes == sorted(sizes), B
    rng = random.Random(H * d + bits)
    for _ in range(3000):
        B, T = int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 17))
        assert size(B, T) >= size(rng.randint(1, B), rng.randint(1, T))


def test_it_does_not_outgrow_the_batch():
    """What is reserved for the splits of smaller batches: less than twice what a batch by itself takes, and no more for one sequence than it took."""
    size = lambda B, T: binding.slim_workspace_bytes_quant(B, 32, T, 4096, 4, "bf16")      # noqa: E731
    for T, one, sixteen in ((777, 7, 16), (16384, 16, 64), (3000, 16, 48)):
        numerators = lambda B: B * 32 * ((T + 63) // 64) * (64 * 2 + 8)      # noqa: E731
        sums = lambda n: n * 32 * (4096 + 2) * 4      # noqa: E731
        assert size(1, T) <= numerators(1) + sums(one) + 16 * 4096 * 4 + (1 << 16)
        assert size(16, T) <= numerators(16) + 2 * sums(sixteen) + 256 * 4096 * 4 + (1 << 16)


@pytest.mark.parametrize("H,d,dtype", WIDTHS)
def test_splits_and_row_splits_have_their_place(H, d, dtype):
    """For every batch, and less than twice what some batch up to it takes."""
    for T in (1, 64, 65, 129, 777, 2049, 5000, 16384, 200000):
        most = most_rows = 0
        for B in range(1, 1200):
            per, splits, row_splits, rows, place, row_place = quant_cut(dtype, B, H, T, d)
            nb = (T + 63) // 64
            assert (splits - 1) * per < nb <= splits * per and splits <= 64
            assert (row_splits - 1) * rows < d <= row_splits * rows and rows <= 256 and rows % 32 == 0
            most, most_rows = max(most, B * splits), max(most_rows, B * row_splits)
            assert most <= place < 2 * most + 1, (B, T)
            assert row_place == 0 if most_rows == B else most_rows <= row_place, (B, T)
