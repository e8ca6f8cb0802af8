"""How prompt attention cuts a call where few sequences of the batch bring queries: parts of the keys for the workgroups that there are, and no more
workgroups than a launch can have.  CPU only."""
import random

import pytest

from launch_rules import prompt_cut


@pytest.mark.parametrize("B,keys", [(16, 4000), (64, 4000), (200, 1500)])
def test_an_idle_sequence_changes_nothing(B, keys):
    """32 heads and one query of each sequence, or of each but one: the chip is full either way, and the keys stay whole."""
    for H_kv, d_k in ((32, 128), (4, 64), (8, 128)):
        for rows_q in (B - 1, B):
            assert prompt_cut("bf16", B, rows_q, B * keys, 32, H_kv, d_k)[1] == 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_are_for_the_sequences_with_queries(dtype):
    """Fewer queries than sequences: as many sequences at the most have any, and are cut as a batch of these alone."""
    for B, busy, keys in ((16, 1, 4000), (16, 5, 4000), (16, 15, 4000), (64, 3, 9000), (64, 63, 600), (300, 40, 2000)):
        for H, H_kv, d_k in ((32, 32, 128), (8, 2, 64)):
            if 4.0 * B * keys * H_kv * d_k <= 1e8:               # (what the last-level cache keeps is told by all keys)
                assert prompt_cut(dtype, B, busy, B * keys, H, H_kv, d_k) == prompt_cut(dtype, busy, busy, busy * keys, H, H_kv, d_k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_launch_has_its_workgroups(dtype):
    """Less than 2^24 workgroups of 256 threads, for every call that is not refused; no parts without queries."""
    rng = random.Random(5)
    cases = [(32768, 1, 1 << 24, 500, 1, 256), (8000, 1, 1 << 24, 2048, 1, 128), (1024, 1023, 1 << 24, 4090, 1, 256), (2000, 7, 1 << 24, 2048, 1, 256), (16408, 1, 1 << 24, 341, 1, 16)]
    for _ in range(4000):
        H = int(2 ** rng.uniform(0, 12))
        cases.append((int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(10, 24)), H, H, rng.choice([8, 64, 128, 256])))
    for B, rows_q, rows_k, H, H_kv, d_k in cases:
        if H * (rows_q // 64 + B + 8) >= 1 << 24:
            continue                                             # (refused)
        rows, parts = prompt_cut(dtype, B, rows_q, rows_k, H, H_kv, d_k)
        places = (rows_q // rows + B + 7) // 8 * 8
        assert places * H * parts < 1 << 24, (B, rows_q, rows_k, H, d_k)
        assert prompt_cut(dtype, B, 0, rows_k, H, H_kv, d_k)[1] == 1
