"""slim_tree_decode over the longest contexts: rows of one sequence past 2^32 bytes, and a batch whose second sequence lies past them, in both layouts."""
import numpy as np
import pytest

from oracle import tree_oracle as orc
from paper_2503_05840_amd import binding, synth
from gpu_harness import say
from tree_cases import HALF, TreeCase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("banded", [False, True])
@pytest.mark.parametrize("H,d_k", [(8, 128), (16, 64)])
def test_rows_past_32_bit_offsets(H, d_k, banded):
    """A context of four million rows, all zero but for forty: a zero row has the score 0 and adds 1 to the softmax sum, nothing else."""
    import torch
    T, N, d = 4190000, 2, 1024
    say(f"[case] tree, {T} rows: H={H} d_k={d_k} banded={banded}")
    rows = (T + N + 31) // 32 * 32
    rng = np.random.default_rng(H)
    at = np.unique(np.concatenate([[0, 255, 256, (1 << 21) - 1, 1 << 21, T - 2, T - 1], rng.integers(0, T, 33)]))
    n = len(at)
    keys = synth.round_through(rng.standard_normal((n + N, d)), "bf16")
    q = synth.round_through(rng.standard_normal((N, d)) * 5.0, "bf16")
    W = synth.round_through(rng.standard_normal((d, d)) / np.sqrt(d), "bf16")
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16)      # noqa: E731
    K = torch.zeros((1, rows, d), dtype=torch.bfloat16, device="cuda")
    places = torch.from_numpy(np.concatenate([at, [T, T + 1]])).cuda()
    if banded:
        K.view(rows // 32, H, 32, d_k)[places // 32, :, places % 32] = up(keys).view(-1, H, d_k)
    else:
        K[0, places] = up(keys)
    parents = torch.tensor([[-1, 0]], dtype=torch.int32, device="cuda")
    out = torch.full((1, N, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    binding.slim_tree_decode(up(q)[None], K, up(W), parents, out, 1, N, H, T, d, t_stride=rows, k_layout=binding.K_BANDED if banded else 0)
    torch.cuda.synchronize()
    got = out.float().cpu().numpy()[0]
    half, f32 = HALF["bf16"], HALF["f32"]
    for i in range(N):
        seen = keys[:n + 1 + i]
        for h in range(H):
            c = slice(h * d_k, (h + 1) * d_k)
            s = seen[:, c] @ q[i, c] / np.sqrt(d_k)
            top = max(s.max(), 0.0)
            p = np.exp(s - top)
            zeros = (T - n) * np.exp(-top)
            z = p.sum() + zeros
            p, rest = p / z, zeros / z
            V = seen @ W[:, c]
            want = p @ V
            spread = p @ np.abs(V - want) + rest * np.abs(want)
            size = (p @ np.abs(seen)) @ np.abs(W[:, c])
            swing = (np.abs(seen[:, c]) @ np.abs(q[i, c])).max() / np.sqrt(d_k)
            # the numerators' rounding, scores and exponentials; sums of forty rows, of the blocks' sums (256 equal ones each: exact) and of d columns in
            # fp32, C as hi + lo; the result's rounding
            blocks = (T + N + 255) // 256
            bound = 1.1 * ((half + (swing * (d_k + 4) + 4) * f32) * spread + size * ((n + N + blocks + d) * f32 + half ** 2) + half * np.abs(want)) + 1e-30
            worst = (np.abs(got[i, c] - want) / bound).max()
            assert worst <= 1.0, (i, h, worst)


def test_a_banded_batch_past_32_bit_offsets():
    """The second sequence's bands lie past 4 GB."""
    import torch
    say("[case] tree, banded cache past 4 GB")
    H, d_k, N, rows = 8, 64, 3, 1 << 22
    c = TreeCase(2, N, H, d_k, 100, "bf16", lens=[100, 60], seed=13, banded=True)
    want = c.run()
    K = torch.zeros((2, rows, H * d_k), dtype=torch.bfloat16, device="cuda")
    K[:, :c.rows] = c.dev["K"]
    out = torch.empty_like(c.dev["q"])
    binding.slim_tree_decode(c.dev["q"], K, c.dev["W"], c.dev["parents"], out, 2, N, H, 100, H * d_k, seq_lens=c.dev["lens"], t_stride=rows,
                             k_layout=binding.K_BANDED)
    torch.cuda.synchronize()
    assert np.array_equal(out.float().cpu().numpy(), want)


@pytest.mark.parametrize("banded", [False, True])
def test_commit_past_32_bit_offsets(banded):
    import torch
    say(f"[case] commit past 4 GB, banded={banded}")
    H, d_k, N, T = 8, 128, 4, 4190000
    d, rows = H * d_k, (T + N + 31) // 32 * 32
    K = torch.zeros((1, rows, d), dtype=torch.bfloat16, device="cuda")
    bands = K.view(rows // 32, H, 32, d_k)
    pick = lambda t: bands[t // 32, :, t % 32].reshape(-1) if banded else K[0, t]      # noqa: E731
    tail = np.random.default_rng(1).standard_normal((N, d)).astype(np.float32)
    for i in range(N):
        row = torch.from_numpy(tail[i]).cuda().to(torch.bfloat16)
        if banded:
            bands[(T + i) // 32, :, (T + i) % 32] = row.view(H, d_k)
        else:
            K[0, T + i] = row
    new = torch.empty(1, dtype=torch.int32, device="cuda")
    binding.slim_tree_commit(K, torch.tensor([[0, 2, 3, -1]], dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda"), new,
                             1, N, H, T, d, t_stride=rows, k_layout=binding.K_BANDED if banded else 0)
    torch.cuda.synchronize()
    assert int(new[0]) == T + 3
    want = orc.commit(tail, [0, 2, 3], 0)
    for i in range(N):
        assert torch.equal(pick(T + i).float().cpu(), torch.from_numpy(want[i]).to(torch.bfloat16).float())
    assert not K[0, :T].any() if not banded else not bands[:T // 32].any()
