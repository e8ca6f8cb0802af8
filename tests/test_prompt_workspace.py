"""slim_workspace_bytes_prompt in all three sizes that change from call to call.  CPU only."""
import itertools
import random

import pytest

from launch_rules import prompt_cut
from paper_2503_05840_amd import binding

HEADS = [(32, 32, 128, "bf16"), (32, 8, 128, "bf16"), (24, 24, 96, "bf16"), (20, 20, 64, "f32"), (24, 24, 64, "f32"), (4, 1, 256, "bf16"), (300, 4, 8, "bf16"),
         (1, 1, 192, "f32")]


@pytest.mark.parametrize("H,H_kv,d_k,dtype", HEADS)
def test_a_smaller_prompt_context_or_batch_never_needs_more(H, H_kv, d_k, dtype):
    size = lambda B, rows_q, rows_k: binding.slim_workspace_bytes_prompt(B, rows_q, rows_k, H, H_kv, d_k, dtype)      # noqa: E731
    queries = sorted({0, 1, 2, 63, 64, 65, 128, 300, 512, 777, 1024, 2048, 4999, 16384} | set(range(5, 1200, 37)))
    keys = sorted({0, 1, 64, 255, 256, 511, 512, 1664, 2064, 8192, 9772, 9836, 16384, 37868, 37932, 200000} | set(range(100, 6000, 113)))
    batches = [1, 2, 3, 4, 5, 15, 16, 17, 63, 64, 200]
    for B, rows_k in itertools.product(batches, keys):
        sizes = [size(B, n, rows_k) for n in queries]
        assert sizes == sorted(sizes), (B, rows_k)
    for B, rows_q in itertools.product(batches, queries):
        sizes = [size(B, rows_q, n) for n in keys]
        assert sizes == sorted(sizes), (B, rows_q)
    rng = random.Random(H * d_k)
    for _ in range(3000):
        B, rows_q, rows_k = rng.randint(1, 300), int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 20))
        assert size(B, rows_q, rows_k) >= size(rng.randint(1, B), rng.randint(0, rows_q), rng.randint(0, rows_k))


@pytest.mark.parametrize("H,H_kv,d_k,dtype", HEADS)
def test_it_holds_the_parts_of_every_call(H, H_kv, d_k, dtype):
    """Partial results and two figures a row, part and head, in fp32; and no more than a bound that the heads' width gives."""
    rng = random.Random(H + d_k)
    cut = 0
    for _ in range(6000):
        B, rows_q, rows_k = int(2 ** rng.uniform(0, 7)), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(6, 21))
        parts = prompt_cut(dtype, B, rows_q, rows_k, H, H_kv, d_k)[1]
        have = binding.slim_workspace_bytes_prompt(B, rows_q, rows_k, H, H_kv, d_k, dtype)
        cut += parts > 1
        if parts > 1:
            assert have >= parts * rows_q * H * (d_k + 2) * 4 + 4096
        assert 0 < have <= 4096 * 129 * (d_k + 2) * 4 + (1 << 16)
    assert cut > 200


def test_the_sizes_that_callers_kept_too_small():
    size = lambda *a, dtype="bf16": binding.slim_workspace_bytes_prompt(*a, dtype)      # noqa: E731
    assert size(1, 16384, 16384, 32, 32, 128) >= size(1, 300, 16384, 32, 32, 128) > 1 << 20
    assert size(1, 1024, 8192, 32, 32, 128) >= size(1, 777, 8192, 32, 32, 128)
    assert size(1, 2048, 8192, 32, 32, 128) >= size(1, 1024, 8192, 32, 32, 128)
    assert size(1, 300, 37932, 24, 24, 64) >= size(1, 300, 37868, 24, 24, 64)
    assert size(1, 256, 2064, 64, 64, 128) >= size(1, 256, 2000, 64, 64, 128)
