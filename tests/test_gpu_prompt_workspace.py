"""One workspace, sized for the largest prompt, context and batch, serves every smaller call and gives the bits of the library's own."""
import numpy as np
import pytest

from launch_rules import prompt_cut
from paper_2503_05840_amd import binding
from prompt_cases import PromptCase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_smaller_calls_on_the_largest_workspace(dtype):
    import torch
    H, H_kv, d_k = 6, 2, 64
    size = binding.slim_workspace_bytes_prompt(8, 9000, 12000, H, H_kv, d_k, dtype)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    cut = 0
    for n_q, n_k in (([1], [9000]), ([130], [4000]), ([700], [2500]), ([3, 1, 0], [900, 2000, 5]), ([300], [300]), ([1] * 8, [1500] * 8)):
        c = PromptCase(n_q, n_k, H, H_kv, d_k, dtype, seed=sum(n_k), tail=1)
        own = c.run()
        got = c.call(workspace=ws)
        torch.cuda.synchronize()
        got = got.float().cpu().numpy().astype(np.float64)
        assert np.array_equal(got, own)
        cut += prompt_cut(dtype, len(n_q), sum(n_q) + 1, sum(n_k) + 1, H, H_kv, d_k)[1] > 1
        if sum(n_q) < 20:
            c.check(got=got)
    assert cut >= 4
