"""slim_tree_decode against the fp64 oracle: types, head widths, lengths from none to several blocks of rows, trees of one node to 64, unused
slots, layouts, rotary positions, values that are not finite in places that a node does not see."""
import numpy as np
import pytest

from paper_2503_05840_amd import binding
from gpu_harness import say
from tree_cases import TreeCase, random_tree

pytestmark = pytest.mark.gpu

SHAPES = [  # (B, N, H, d_k, T, dtype, lens, base, banded)
    (1, 1, 1, 8, 0, "bf16", None, None, False), (1, 1, 4, 64, 1, "bf16", None, None, False), (1, 1, 1, 4, 0, "f32", None, None, False),
    (2, 5, 8, 64, 40, "bf16", [40, 0], None, False), (3, 13, 4, 64, 300, "f32", [300, 1, 255], None, False),
    (1, 64, 2, 128, 200, "bf16", None, None, False), (1, 64, 2, 32, 448, "f32", None, 10000.0, False),
    (2, 16, 8, 96, 261, "bf16", [261, 240], 10000.0, False), (2, 7, 20, 64, 224, "bf16", [224, 31], None, True),
    (2, 21, 5, 80, 700, "bf16", [100, 700], 500.0, True), (1, 33, 3, 72, 1025, "bf16", None, None, False),
    (2, 3, 40, 16, 513, "bf16", [512, 513], None, False), (1, 2, 3, 136, 90, "bf16", None, None, False), (1, 17, 2, 260, 70, "f32", None, None, False),
    (5, 11, 6, 24, 255, "f32", [255, 254, 253, 0, 7], None, True), (17, 4, 3, 8, 33, "bf16", list(range(17)), 10000.0, False),
    (1, 9, 130, 8, 64, "bf16", None, None, False), (1, 63, 16, 8, 1990, "bf16", None, None, False),
]


@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_against_the_oracle(i):
    B, N, H, d_k, T, dtype, lens, base, banded = SHAPES[i]
    say(f"[case] tree: B={B} N={N} H={H} d_k={d_k} T={T} {dtype} base={base} banded={banded}")
    c = TreeCase(B, N, H, d_k, T, dtype, lens=lens, base=base, banded=banded, seed=100 + i, slack=3 * (i % 3))
    say(f"       {c.check():.3f} of the bound")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unused_slots_are_zero_and_change_nothing(dtype):
    """Bad parents, their descendants, several roots; the used nodes' results are those of the tree without the others."""
    N = 12
    par = [-1, 0, -2, 2, 1, 5, 99, -1, 7, 3, 8, -2147483648]        # 2, 3, 5 (itself), 6, 9, 11 are unused
    say(f"[case] tree with unused slots, {dtype}")
    c = TreeCase(1, N, 4, 32, 50, dtype, parents=par, seed=7)
    got = c.run()
    c.check(got)
    for i in (2, 3, 5, 6, 9, 11):
        assert (got[0, i] == 0).all()
    c.K[0, [52, 53, 55, 56, 59, 61]] = np.nan                       # (their keys are seen by nobody)
    assert np.array_equal(c.run(), got)
    c.parents[:] = -5
    assert (c.run() == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_keys_that_are_not_finite_reach_only_the_nodes_that_see_them(dtype, value):
    N, T = 10, 30
    par = [-1, 0, 0, 1, 1, 2, 3, 2, 5, 0]
    say(f"[case] tree, drafted key {value}, {dtype}")
    c = TreeCase(2, N, 4, 64, T, dtype, lens=[T, T - 9], parents=[par, par], seed=9, slack=70)
    clean = c.run()
    c.K[0, T + 2, 5] = value                                        # nodes 2, 5, 7, 8 see it
    c.K[:, T + N:] = value                                          # rows past the drafted ones: nobody
    got = c.run()
    sees = [2, 5, 7, 8]
    assert not np.isfinite(got[0, sees]).any()
    others = [i for i in range(N) if i not in sees]
    assert np.array_equal(got[0, others], clean[0, others]) and np.array_equal(got[1], clean[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_apart(dtype):
    """Queries large enough that a few rows take all the weight and references of the row blocks differ by many steps."""
    say(f"[case] tree, far scores, {dtype}")
    c = TreeCase(1, 6, 4, 64, 1500, dtype, seed=11, q_scale=60.0)
    c.check()
    c.K[0, :600] *= 0.01
    c.K[0, 600:900] *= 0.1
    from paper_2503_05840_amd import synth
    c.K = synth.round_through(c.K, dtype)
    c.check()
    c.K[0, :1500] = c.K[0, :1500][::-1]
    c.check()


def test_a_long_cache_past_32_bit_offsets():
    """A cache of more than 2^32 bytes: the second sequence's rows lie past it, in both layouts."""
    import torch
    say("[case] tree, cache past 4 GB")
    H, d_k, N, rows = 8, 64, 3, 1 << 22
    c = TreeCase(2, N, H, d_k, 100, "bf16", lens=[100, 60], seed=13)
    want = c.run()
    K = torch.zeros((2, rows, H * d_k), dtype=torch.bfloat16, device="cuda")
    K[:, :103] = c.dev["K"]
    out = torch.empty_like(c.dev["q"])
    binding.slim_tree_decode(c.dev["q"], K, c.dev["W"], c.dev["parents"], out, 2, N, H, 100, H * d_k, seq_lens=c.dev["lens"], t_stride=rows)
    torch.cuda.synchronize()
    assert np.array_equal(out.float().cpu().numpy(), want)


def test_workspace_stream_and_graph():
    """A caller's workspace of exactly the stated size on another stream, and a captured call replayed with other inputs, give the eager bits."""
    import torch
    say("[case] tree, workspace, stream, graph")
    c = TreeCase(2, 9, 8, 64, 300, "bf16", lens=[300, 120], seed=17)
    want = c.run()
    n = binding.slim_workspace_bytes_tree(2, 9, 8, 300, 512, "bf16")
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(c.dev["q"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.call(out=out, workspace=ws[:n])
    torch.cuda.synchronize()
    assert np.array_equal(out.float().cpu().numpy(), want)
    assert (ws[n:] == 255).all()
    with pytest.raises(binding.SlimError):
        c.call(out=out, workspace=ws[:n - 256])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.call(out=out, workspace=ws[:n])
    q0 = c.dev["q"].clone()
    for k in range(4):
        c.dev["q"].copy_(q0 * (1.0 - 0.25 * k))
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        c.call(out=out)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.isfinite(out).all()


@pytest.mark.parametrize("N", [1, 4])
def test_a_chain_gives_what_single_steps_give(N):
    """A tree without branches is N generation steps: slim_decode's results, one row of the cache after the other."""
    import torch
    say(f"[case] tree against single steps, N={N}")
    c = TreeCase(1, N, 8, 64, 200, "f32", parents=[list(range(-1, N - 1))], seed=19)
    got = c.run()
    one = torch.empty((1, c.d), device="cuda")
    for i in range(N):
        K = c.dev["K"][:, :201 + i].contiguous()
        binding.slim_decode(c.dev["q"][:, i].contiguous(), K, c.dev["W"], one, 1, 8, 201 + i, c.d, dtype="f32")
        torch.cuda.synchronize()
        want = one.cpu().numpy()[0]
        # both within the oracle's bound; sums of 700 terms in another order
        assert np.abs(got[0, i] - want).max() <= 2 * 700 * 2.0 ** -24 * 8


MANY_BLOCKS = [  # (B, N, H, d_k, T, dtype, lens, base, banded): enough workgroups of scores for those that walk over row blocks or heads, splits of ragged batches
    (4, 3, 16, 64, 2300, "f32", [2300, 700, 1, 1999], None, False), (2, 5, 16, 104, 4400, "bf16", None, None, False),
    (4, 3, 64, 8, 1100, "bf16", [1100, 0, 255, 1024], 10000.0, False), (3, 16, 72, 16, 1250, "bf16", [513, 1250, 767], 10000.0, True),
    (5, 2, 64, 4, 1000, "f32", [3, 1000, 511, 512, 800], 500.0, False), (9, 6, 8, 32, 3000, "bf16", [40, 3000, 0, 700, 64, 2222, 1, 333, 2900], None, False),
    (70, 1, 2, 8, 900, "f32", [(37 * i) % 901 for i in range(70)], None, False),
]


@pytest.mark.parametrize("i", range(len(MANY_BLOCKS)))
def test_many_row_blocks_against_the_oracle(i):
    B, N, H, d_k, T, dtype, lens, base, banded = MANY_BLOCKS[i]
    say(f"[case] tree, many blocks: B={B} N={N} H={H} d_k={d_k} T={T} {dtype} base={base} banded={banded}")
    c = TreeCase(B, N, H, d_k, T, dtype, lens=lens, base=base, banded=banded, seed=300 + i)
    say(f"       {c.check():.3f} of the bound")


@pytest.mark.parametrize("B,N,H,d_k,T,dtype,base", [(1, 5, 16, 64, 40, "bf16", None), (4, 5, 16, 64, 2300, "f32", None), (4, 5, 64, 8, 1100, "bf16", 10000.0)])
def test_a_context_that_is_not_finite_leaves_unused_slots_zero(B, N, H, d_k, T, dtype, base):
    say(f"[case] tree, NaN in the context: B={B} N={N} H={H} d_k={d_k} T={T} {dtype}")
    c = TreeCase(B, N, H, d_k, T, dtype, parents=[[-1, 0, 7, 0, 2]] * B, base=base, seed=23)
    c.K[:, 5] = np.nan
    c.K[0, T - 1] = np.inf
    got = c.run()
    assert (got[:, [2, 4]] == 0).all() and not np.isfinite(got[:, [0, 1, 3]]).any()
