"""Prompt attention over batches in which some sequences bring no queries."""
import numpy as np
import pytest

from launch_rules import prompt_cut
from paper_2503_05840_amd import binding
from prompt_cases import PromptCase, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_k,H,d_k", [([1, 0, 1, 1], [900, 700, 5, 2000], 4, 64), ([0, 0, 1, 0, 0], [10, 0, 3000, 40, 0], 2, 128),
                                           ([1] * 15 + [0], [300 + 20 * b for b in range(16)], 32, 32)])
def test_fewer_queries_than_sequences(n_q, n_k, H, d_k, dtype, causal):
    PromptCase(n_q, n_k, H, H, d_k, dtype, causal, seed=sum(n_k)).check()


def test_keys_stay_whole_where_all_sequences_but_one_fill_the_chip():
    """Nothing is left in the workspace."""
    import torch
    B, keys, H, H_kv, d_k = 16, 4000, 32, 1, 64
    c = PromptCase([1] * (B - 1) + [0], [keys] * B, H, H_kv, d_k, seed=1)
    c.device()
    ws = torch.full((1 << 28,), 0xa5, dtype=torch.uint8, device="cuda")
    got = c.call(workspace=ws)
    torch.cuda.synchronize()
    assert (ws == 0xa5).all()
    c.check(got=got.float().cpu().numpy().astype(np.float64), sequences=[0, 14])


def test_more_places_than_a_launch_has_for_parts():
    """16408 sequences x 341 heads, of which one sequence has a query: alone its keys are cut, and with the others' places its parts would be more workgroups than a
    launch can have."""
    import torch
    B, H, d_k, rows_k = 16408, 341, 16, 1 << 24
    parts = prompt_cut("f32", 1, 1, rows_k // B, H, 1, d_k)[1]
    assert parts > 1 and B * H * parts >= 1 << 24 and prompt_cut("f32", B, 1, rows_k, H, 1, d_k)[1] == 1
    kv = torch.ones((rows_k, d_k), device="cuda")
    q = torch.ones((1, H * d_k), device="cuda")
    out = torch.full_like(q, 77.0)
    b = 9000
    binding.slim_prompt_attention(q, kv, kv, ints([0] * (b + 1) + [1] * (B - b)), out, B, H, 1, d_k,
                                  cu_k=ints(np.arange(B + 1) * (rows_k // B)), dtype="f32")
    torch.cuda.synchronize()
    # Equal numerators, of which the weighted sum and the sum differ by their order alone: half a step an addition, in both
    assert ((out - 1).abs() <= 2 * (rows_k // B + 4) * 2.0 ** -24).all()
