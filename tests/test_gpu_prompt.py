"""Attention over whole prompts against fp64: types, head layouts, lengths, masks, and what lies in masked places."""
import numpy as np
import pytest

from paper_2503_05840_amd import binding
from prompt_cases import PromptCase, ints, offsets, up

pytestmark = pytest.mark.gpu

SHAPES = [  # n_q, n_k, H, H_kv, d_k
    ([1], [1], 1, 1, 64), ([63], [63], 2, 2, 128), ([128], [128], 2, 1, 96), ([129, 1, 0, 64], [129, 1, 0, 64], 4, 2, 64), ([33], [200], 3, 1, 80),
    ([5, 40], [5, 300], 2, 2, 112), ([70], [30], 2, 2, 64), ([200], [200], 1, 1, 32), ([65], [65], 2, 2, 40), ([90], [90], 2, 1, 192), ([100], [131], 1, 1, 256),
    ([0, 17, 0], [4, 17, 0], 2, 2, 72), ([3, 9], [0, 9], 2, 2, 64), ([150], [150], 1, 1, 128), ([16], [16], 2, 2, 8), ([1, 1, 1], [66, 1, 64], 4, 4, 128)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_k,H,H_kv,d_k", SHAPES)
def test_against_fp64(n_q, n_k, H, H_kv, d_k, dtype, causal):
    PromptCase(n_q, n_k, H, H_kv, d_k, dtype, causal, seed=sum(n_k) + d_k, tail=3).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv", [(9, 9), (20, 20), (7, 1), (24, 12), (26, 13)])
def test_heads_that_do_not_share_out_evenly(dtype, H, H_kv):
    """Every head and tile is somebody's, whatever is left over the eight XCDs."""
    PromptCase([260, 70, 5], [260, 70, 5], H, H_kv, 32, dtype, seed=H).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
def test_no_keys_at_all_and_rows_before_the_first_sequence(dtype, causal):
    import torch
    c = PromptCase([3], [0], 2, 2, 64, dtype, causal)
    assert (c.run() == 0).all()
    c = PromptCase([40, 90], [40, 90], 2, 1, 64, dtype, causal, seed=1)
    want = c.run()
    cut = 7                                                      # the first sequence starts seven rows later
    c.dev["cu_q"] = ints([cut, 40, 130])
    got = c.call().float().cpu().numpy()
    assert (got[:cut] == 77.0).all() and np.array_equal(got[40:], want[40:])
    d = PromptCase([40 - cut], [40 - cut], 2, 1, 64, dtype, causal)
    d.q, d.k, d.v = c.q[cut:40], c.k[cut:40], c.v[cut:40]
    assert np.array_equal(got[cut:40], d.run())
    torch.cuda.synchronize()


@pytest.mark.parametrize("d_k", [4, 36, 100, 180, 252])
def test_widths_of_fp32_vectors(d_k):
    PromptCase([70, 5], [70, 5], 2, 1, d_k, "f32", seed=d_k).check()


@pytest.mark.parametrize("dtype,H,H_kv,d_k", [("bf16", 16, 2, 128), ("f32", 2, 2, 64)])
def test_many_sequences(dtype, H, H_kv, d_k):
    lens = [1 + (b * 37) % 70 for b in range(40)]
    PromptCase(lens, lens, H, H_kv, d_k, dtype, seed=8, tail=1).check(sequences=[0, 1, 17, 39])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_k,H", [([1], [4000], 2), ([20, 3], [3000, 900], 2), ([100], [2500], 1), ([1, 1], [5000, 1], 4)])
def test_few_queries_over_many_keys(dtype, n_q, n_k, H):
    """Keys shared out over workgroups, causal and full."""
    for causal in (True, False):
        c = PromptCase(n_q, n_k, H, H, 64, dtype, causal, seed=5, tail=2)
        whole = binding.slim_workspace_bytes_prompt(len(n_q), c.q.shape[0], c.q.shape[0], H, H, 64, dtype)
        assert binding.slim_workspace_bytes_prompt(len(n_q), c.q.shape[0], c.k.shape[0], H, H, 64, dtype) > whole       # (in parts)
        c.check()


def test_long_prompt():
    rows = [0, 1, 2047, 2048, 4095, 4999]
    PromptCase([5000], [5000], 2, 1, 128, seed=1).check(queries=rows)


def test_scores_far_apart():
    """References that move often, and numerators far below them."""
    for dtype in ("bf16", "f32"):
        PromptCase([300], [300], 2, 2, 64, dtype, seed=7, q_scale=40.0).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
def test_what_is_not_seen_has_no_effect(dtype, causal):
    """Keys and values behind a query's last key, and rows of no sequence, hold NaN and infinities."""
    n = 150
    c = PromptCase([n], [n], 2, 1, 96, dtype, causal, seed=3, tail=70)
    clean = c.run()[:n]
    c.k[n:], c.v[n:] = np.nan, np.inf
    if causal:
        for row, x in ((100, np.nan), (101, np.inf), (149, -np.inf)):
            c.v[row, 3::7] = x
        c.k[130] = np.inf
        c.k[140] = np.nan
    got = c.run()[:n]
    if not causal:
        assert np.array_equal(got, clean)
        return
    assert np.array_equal(got[:100], clean[:100])
    bad = np.zeros((n, 96), dtype=bool)
    bad[100:, 3::7] = True
    bad[140:] = True                                             # (a key that is NaN makes every column NaN)
    bad = np.tile(bad, (1, 2))
    sees_inf = np.zeros_like(bad)
    sees_inf[130:] = True                                        # (an infinite key: NaN, or nothing where its score is -inf)
    assert not np.isfinite(got[bad]).any()
    ok = ~bad & ~sees_inf
    assert np.isfinite(got[ok]).all() and np.allclose(got[ok], clean[ok], rtol=2.0 ** -6, atol=2.0 ** -6)


def test_columns_of_one_buffer():
    import torch
    c = PromptCase([77, 130], [77, 130], 4, 2, 64, seed=2)
    want = c.run()
    wide = torch.cat([c.dev["q"], c.dev["k"], c.dev["v"]], 1)
    e = 4 * 64
    c.dev.update(q=wide[:, :e], k=wide[:, e:e + 128], v=wide[:, e + 128:])
    assert np.array_equal(c.call().float().cpu().numpy(), want)
    one = up(np.ones((1, e)), "bf16")
    c.dev["k"] = one[:, :128].expand(207, 128)
    with pytest.raises(ValueError):
        c.call()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_past_32_bit_offsets(dtype):
    """Columns of a buffer of 2^20 columns a row: rows from 2048 on are past 2^31 elements."""
    import torch
    n, e = 2200, 2 * 64
    c = PromptCase([n], [n], 2, 2, 64, dtype, seed=9)
    want = c.run()
    wide = torch.zeros((n, 1 << 20), dtype=c.dev["q"].dtype, device="cuda")
    for i, name in enumerate(("q", "k", "v")):
        at = slice((1 << 20) - (i + 1) * e, (1 << 20) - i * e)
        wide[:, at] = c.dev[name]
        c.dev[name] = wide[:, at]
    assert np.array_equal(c.call().float().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_that_are_out_of_range_stay_inside(dtype):
    """Offsets are device data: whatever they are, only rows that there are get read and written."""
    import torch
    c = PromptCase([50, 50], [50, 50], 2, 2, 64, dtype, seed=6)
    c.device()
    for cu in ([0, 50, 5000], [-7, 50, 100], [90, 10, 100], [100, 0, 0], [1 << 30, 1 << 30, 1 << 30]):
        c.dev["cu_q"] = ints(cu)
        c.call()
    torch.cuda.synchronize()
    c.dev["cu_q"] = ints([0, 50, 5000])
    assert np.array_equal(c.call().float().cpu().numpy(), c.run())


def test_the_same_bits_on_dirty_scratch_and_other_streams():
    import torch
    c = PromptCase([9], [3000], 2, 2, 128, seed=4)
    c.device()
    ws = torch.full((binding.slim_workspace_bytes_prompt(1, 9, 3000, 2, 2, 128, "bf16"),), 0xff, dtype=torch.uint8, device="cuda")
    a, own = c.call(workspace=ws), c.call()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        other = c.call(workspace=torch.zeros_like(ws))
    torch.cuda.synchronize()
    assert torch.equal(a, own) and torch.equal(a, other)
    graph = torch.cuda.CUDAGraph()
    out = torch.empty_like(a)
    with torch.cuda.graph(graph):
        c.call(out=out, workspace=ws)
    for i in range(3):
        c.dev["q"].mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        want = c.call()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


def test_prompt_cache_and_generation_together():
    """A prompt taken in two pieces, its keys kept in 8 bits and read back for the second piece, then generated tokens: against fp64 on the values that
    the cache holds, step by step."""
    import torch
    from oracle import prompt_oracle as orc
    from oracle import tree_oracle
    rng = np.random.default_rng(11)
    B, H, d_k, bits = 2, 4, 64, 8
    d = H * d_k
    lens, first, steps = [90, 133], [50, 70], 3
    T = 140
    W = up(rng.standard_normal((d, d)) / np.sqrt(d), "bf16")
    codes, scales = binding.slim_quant_cache(B, T, d, bits)
    held = [0, 0]
    stored = [np.zeros((0, d)), np.zeros((0, d))]
    for piece in (first, [a - b for a, b in zip(lens, first)]):
        n = sum(piece)
        k, q = (up(rng.standard_normal((n, d)) * f, "bf16") for f in (1.0, 1.5))
        cu, at = ints(offsets(piece)), offsets(piece)
        binding.slim_quant_append(k, codes, scales, B, T, d, bits, cu_rows=cu, seq_lens=ints(held))
        now = [h + p for h, p in zip(held, piece)]
        cu_k = ints(offsets(now))
        keys = torch.empty((sum(now), d), dtype=torch.bfloat16, device="cuda")
        binding.slim_quant_read(codes, scales, keys, B, T, d, bits, cu_rows=cu_k)
        values = (keys.float() @ W.float()).bfloat16()            # what the cache's rows stand for in the steps to come
        out = torch.empty_like(q)
        binding.slim_prompt_attention(q, keys, values, cu, out, B, H, H, d_k, cu_k=cu_k)
        at_k = offsets(now)
        for b in range(B):
            c, s = orc.quantise(k[at[b]:at[b + 1]].double().cpu().numpy(), bits)
            stored[b] = np.concatenate([stored[b], orc.values(c, s, bits)])
            assert np.array_equal(stored[b], keys[at_k[b]:at_k[b + 1]].double().cpu().numpy())
            o, spread, size, swing = orc.prompt_attention(q[at[b]:at[b + 1]].double().cpu().numpy(), stored[b],
                                                          values[at_k[b]:at_k[b + 1]].double().cpu().numpy(), H, H, True)
            got = out[at[b]:at[b + 1]].double().cpu().numpy()
            assert (np.abs(got - o) <= 1.1 * (2.0 ** -8 * (size + np.abs(o)) + 1e-4 * spread)).all()
        held = now
    for _ in range(steps):
        k, q = (up(rng.standard_normal((B, d)) * f, "bf16") for f in (1.0, 1.2))
        binding.slim_quant_append(k, codes, scales, B, T, d, bits, seq_lens=ints(held))
        held = [h + 1 for h in held]
        out = torch.empty_like(q)
        binding.slim_quant_decode(q, codes, scales, W, out, B, H, T, d, bits, seq_lens=ints(held))
        for b in range(B):
            c, s = orc.quantise(k[b:b + 1].double().cpu().numpy(), bits)
            stored[b] = np.concatenate([stored[b], orc.values(c, s, bits)])
            o, spread, size, _ = tree_oracle.tree_attention(q[b:b + 1].double().cpu().numpy(), stored[b], W.double().cpu().numpy(), [-1], held[b] - 1, H)
            got = out[b].double().cpu().numpy()
            assert (np.abs(got - o[0]) <= 1.1 * (2.0 ** -8 * (spread[0] + np.abs(o[0])) + 1e-4 * size[0])).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n_q,n_k,H,H_kv,d_k", [
    ([150, 129, 1], [150, 129, 1], 512, 8, 128), ([129, 128], [129, 128], 512, 512, 32), ([140], [140], 512, 8, 40), ([150, 64], [260, 64], 512, 8, 64),
    ([150, 0], [100, 50], 640, 4, 80), ([140], [140], 512, 8, 96)])
def test_prompts_that_fill_the_chip(n_q, n_k, H, H_kv, d_k, causal):
    """So many heads that a workgroup has 128 queries, where it has 64 with fewer."""
    PromptCase(n_q, n_k, H, H_kv, d_k, "bf16", causal, seed=H + d_k, tail=3).check()


def test_what_is_not_seen_has_no_effect_where_the_chip_is_full():
    """As above, with 128 queries a workgroup."""
    n, H, d_k = 150, 1024, 96
    c = PromptCase([n], [n], H, 8, d_k, "bf16", True, seed=4, tail=70)
    clean = c.run()[:n].reshape(n, H, d_k)
    c.k[n:], c.v[n:] = np.nan, np.inf
    for row, x in ((100, np.nan), (101, np.inf), (149, -np.inf)):
        c.v[row] = x
    got = c.run()[:n].reshape(n, H, d_k)
    assert np.array_equal(got[:100], clean[:100])
    assert not np.isfinite(got[100:]).any()


def test_the_same_sequence_among_few_and_many_heads():
    """64 and 128 queries a workgroup differ by the order of their sums alone: each keeps its bound, and heads of one call are alike whatever the others are."""
    few = PromptCase([300], [300], 4, 4, 64, "bf16", True, seed=12)
    a = few.run()
    few.check(a)
    many = PromptCase([300], [300], 1024, 4, 64, "bf16", True, seed=12)
    many.k, many.v = few.k, few.v
    many.q = np.repeat(few.q.reshape(300, 4, 64), 256, axis=1).reshape(300, 1024 * 64)
    b = many.run().reshape(300, 4, 256, 64)
    assert (b == b[:, :, :1]).all()
    want, bound = few.expected(0)
    assert (np.abs(b[:, :, 0].reshape(300, 256) - want) <= bound).all()
