"""A step of a model with several layers: every layer's commit takes the lengths of before the step, and the last one's writes the new ones in their place."""
import numpy as np
import pytest

from oracle import tree_oracle as orc
from paper_2503_05840_amd import binding
from gpu_harness import say

pytestmark = pytest.mark.gpu


def test_commit_layer_by_layer():
    import torch
    say("[case] commit: three layers")
    rng = np.random.default_rng(5)
    layers, B, N, H, d, T = 3, 2, 6, 2, 32, 20
    K = rng.standard_normal((layers, B, T + N, d)).astype(np.float32)
    lens = np.array([20, 7], dtype=np.int32)
    paths = [[0, 2, 5], [0, 1, 3, 4]]
    path = np.array([p + [-1] * (N - len(p)) for p in paths], dtype=np.int32)
    up = lambda a: torch.from_numpy(a).cuda()      # noqa: E731
    Kd, ld, pd, nd = up(K), up(lens), up(path), up(np.array([len(p) for p in paths], dtype=np.int32))
    elsewhere = torch.empty_like(ld)
    for i in range(layers):
        binding.slim_tree_commit(Kd[i], pd, nd, ld if i + 1 == layers else elsewhere, B, N, H, T, d, dtype="f32", seq_lens=ld)
    torch.cuda.synchronize()
    want = np.stack([[orc.commit(K[i, b], paths[b], int(lens[b])) for b in range(B)] for i in range(layers)])
    assert np.array_equal(Kd.cpu().numpy(), want)
    assert list(ld.cpu().numpy()) == list(elsewhere.cpu().numpy()) == [23, 11]
