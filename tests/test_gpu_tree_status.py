"""A workspace that decode steps and drafted trees share: the control block at its start, which holds what slim_status reads, is the decode step's."""
import numpy as np
import pytest

from paper_2503_05840_amd import binding, synth
from gpu_harness import KCase, say
from tree_cases import TreeCase

pytestmark = pytest.mark.gpu

CONTROL_BYTES = 16384


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,H,d_k,T", [(1, 16, 4, 32, 700), (5, 64, 2, 64, 300), (1, 1, 1, 8, 0)])
def test_the_control_block_is_left_alone(B, N, H, d_k, T, dtype):
    import torch
    say(f"[case] tree, control block: B={B} N={N} H={H} d_k={d_k} T={T} {dtype}")
    c = TreeCase(B, N, H, d_k, T, dtype, seed=41)
    c.device()
    ws = torch.empty(binding.slim_workspace_bytes_tree(B, N, H, T, c.d, dtype) // 4 + CONTROL_BYTES, dtype=torch.int32, device="cuda")
    before = torch.arange(CONTROL_BYTES // 4, dtype=torch.int32, device="cuda") * 1000003 + 12345
    ws[:CONTROL_BYTES // 4] = before
    c.call(workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(ws[:CONTROL_BYTES // 4], before)


def test_a_time_out_is_still_reported_after_a_tree_and_none_is_invented():
    import torch
    cfg = synth.scaled(synth.CONFIGS[1], T=8192)
    k = KCase(cfg, need_v=False)
    c = TreeCase(1, 16, 4, 32, 700, "bf16", seed=43)
    c.q[:] = 0.0                                            # (all numerators are alike)
    c.device()
    need = max(binding.slim_workspace_bytes(cfg.B, cfg.H, cfg.T, cfg.d, "bf16"), binding.slim_workspace_bytes_tree(1, 16, 4, 700, c.d, "bf16"))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    binding.slim_init()
    say("[case] tree, status: ordinary decode, tree")
    k.run_slim(workspace=ws)
    c.call(workspace=ws)
    assert binding.slim_status(ws) == binding.SLIM_OK
    say("[case] tree, status: decode without any waiting, tree")
    assert np.isnan(k.run_slim(workspace=ws, wait_budget_us=-1)).all()
    c.call(workspace=ws)
    assert binding.slim_status(ws) == binding.SLIM_ERR_TIMEOUT
