"""One workspace, sized for the largest batch and context, serves every smaller decode step over a cache in 4 or 8 bits and gives the bits of the library's own."""
import numpy as np
import pytest

from launch_rules import quant_cut
from paper_2503_05840_amd import binding
from prompt_cases import QuantCase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,d_k", [("bf16", 20, 64), ("f32", 9, 32)])
def test_smaller_batches_on_the_largest_workspace(dtype, H, d_k):
    import torch
    B, T, d = 9, 1500, H * d_k
    ws = torch.full((binding.slim_workspace_bytes_quant(B, H, T, d, 4, dtype),), 0xff, dtype=torch.uint8, device="cuda")
    cuts = set()
    for b, t in ((9, 1500), (8, 1500), (3, 777), (1, 1500), (1, 1)):
        c = QuantCase(b, H, d_k, t, 4, dtype, lens=[max(t - 91 * i, 0) for i in range(b)], seed=t + b)
        own = c.run()
        got = c.call(workspace=ws)
        torch.cuda.synchronize()
        got = got.float().cpu().numpy().astype(np.float64)
        assert np.array_equal(got, own)
        c.check(got=got, sequences=[0, b - 1])
        cuts.add(quant_cut(dtype, b, H, t, d)[1:3])
    assert len(cuts) >= 3
