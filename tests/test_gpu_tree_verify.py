"""slim_tree_verify and slim_tree_commit against the fp64 oracle: every output is a whole number or a moved row, so all of them are equal."""
import numpy as np
import pytest

from oracle import tree_oracle as orc
from paper_2503_05840_amd import binding, synth
from gpu_harness import say
from tree_cases import random_tree

pytestmark = pytest.mark.gpu


def _probabilities(rng, B, N, V, dtype, draft):
    logits = rng.standard_normal((B, N, V)) * 3.0
    soft = lambda x: np.exp(x - x.max(-1, keepdims=True)) / np.exp(x - x.max(-1, keepdims=True)).sum(-1, keepdims=True)  # noqa: E731
    p = synth.round_through(soft(logits), dtype)
    q = synth.round_through(soft(logits + rng.standard_normal((B, N, V)) * 0.7), dtype)
    return p, q


def _call(tokens, parents, p, q, u, dtype, stream=None):
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    up = lambda a, ty: torch.from_numpy(np.ascontiguousarray(a)).cuda().to(ty)  # noqa: E731
    B, N, V = p.shape
    dev = (up(tokens, torch.int32), up(parents, torch.int32), up(p.astype(np.float32), t), None if q is None else up(q.astype(np.float32), t),
           up(u, torch.float32))
    path, n_path, nxt = (torch.full(s, -77, dtype=torch.int32, device="cuda") for s in ((B, N), (B,), (B,)))
    binding.slim_tree_verify(*dev, path, n_path, nxt, B, N, V, dtype=dtype)
    torch.cuda.synchronize()
    return path.cpu().numpy(), n_path.cpu().numpy(), nxt.cpu().numpy()


def _same(got, tokens, parents, p, q, u):
    path, n_path, nxt = got
    for b in range(p.shape[0]):
        want, v = orc.verify(tokens[b], parents[b], p[b], None if q is None else q[b], u[b])
        assert n_path[b] == len(want), (b, n_path[b], want)
        assert list(path[b]) == want + [-1] * (p.shape[1] - len(want)), (b, path[b], want)
        assert nxt[b] == v, (b, nxt[b], v)


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,V", [(1, 1, 1), (3, 4, 7), (5, 8, 1000), (2, 64, 4099), (9, 13, 257), (1, 5, 70001)])
def test_walk_and_next_token(B, N, V, dtype, draft):
    say(f"[case] verify: B={B} N={N} V={V} {dtype} draft={draft}")
    rng = np.random.default_rng(B * 1000 + N + V)
    for k in range(3):
        p, q = _probabilities(rng, B, N, V, dtype, draft)
        parents = np.stack([random_tree(rng, N, used=int(rng.integers(1, N + 1)), deep=k == 1) for _ in range(B)])
        tokens = np.zeros((B, N), dtype=np.int32)
        for b in range(B):
            for i in range(N):
                row = q[b, max(0, parents[b, i])]
                tokens[b, i] = rng.choice(V, p=row / row.sum()) if k < 2 else rng.integers(0, min(V, 4))
        u = rng.random((B, N)).astype(np.float32)
        _same(_call(tokens, parents, p, q if draft else None, u, dtype), tokens, parents, p, q if draft else None, u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_borders(dtype):
    """Random numbers of 0 and just under 1, probabilities of 0 and 1, tokens outside the vocabulary, a draft that is the target, a
    residual with nothing left."""
    say(f"[case] verify: borders, {dtype}")
    V, N = 300, 5
    p = np.zeros((6, N, V))
    p[:, :, 17] = 0.5
    p[:, :, 250] = 0.25
    p[:, :, 251] = 0.25
    q = p.copy()
    parents = np.tile(np.array([-1, 0, 0, 1, 3], dtype=np.int32), (6, 1))
    tokens = np.tile(np.array([0, 17, 250, 251, 17], dtype=np.int32), (6, 1))
    u = np.full((6, N), 0.25, dtype=np.float32)
    u[1] = 0.0
    u[2] = np.float32(1) - np.float32(2 ** -24)
    tokens[3] = [0, -1, V, 1 << 30, 17]
    tokens[4] = [0, 5, 6, 7, 8]                             # the target gives them nothing, and neither does the draft
    q[5] = 0.0
    q[5, :, 17] = 1.0                                       # a draft that always proposes 17
    u[5] = [0.75, 0.9, 0.4, 0.1, 0.1]
    _same(_call(tokens, parents, p, q, u, dtype), tokens, parents, p, q, u)
    _same(_call(tokens, parents, p, None, u, dtype), tokens, parents, p, None, u)
    p[0] = 0.0                                              # no probability anywhere: the lowest token
    q[1] = 2 * p[1]                                         # rejected, and nothing is left: the likeliest
    u[1] = 0.75
    _same(_call(tokens, parents, p, q, u, dtype), tokens, parents, p, q, u)


@pytest.mark.parametrize("banded", [False, True])
@pytest.mark.parametrize("B,N,H,d_k,T,dtype", [(1, 1, 1, 8, 0, "bf16"), (3, 8, 8, 64, 50, "bf16"), (2, 64, 20, 64, 90, "bf16"), (2, 13, 5, 24, 31, "f32"),
                                               (1, 9, 70, 128, 40, "f32")])
def test_commit(B, N, H, d_k, T, dtype, banded):
    import torch
    say(f"[case] commit: B={B} N={N} H={H} d_k={d_k} T={T} {dtype} banded={banded}")
    rng = np.random.default_rng(N + T)
    d, rows = H * d_k, (T + N + 31) // 32 * 32
    K = synth.round_through(rng.standard_normal((B, rows, d)), dtype).astype(np.float32)
    lens = rng.integers(0, T + 1, size=B).astype(np.int32)
    paths = [sorted(rng.choice(N, size=int(rng.integers(1, N + 1)), replace=False)) for _ in range(B)]
    paths = [sorted({0, *map(int, p)}) for p in paths]
    path = np.full((B, N), -1, dtype=np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    lay = (lambda x: x.reshape(B, rows // 32, 32, H, d_k).transpose(0, 1, 3, 2, 4).reshape(B, rows, d)) if banded else (lambda x: x)
    Kd = torch.from_numpy(np.ascontiguousarray(lay(K))).cuda().to(t)
    ld, pd = torch.from_numpy(lens).cuda(), torch.from_numpy(path).cuda()
    nd = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    binding.slim_tree_commit(Kd, pd, nd, ld, B, N, H, T, d, dtype=dtype, seq_lens=ld, t_stride=rows, k_layout=binding.K_BANDED if banded else 0)
    torch.cuda.synchronize()
    want = np.stack([orc.commit(K[b], paths[b], int(lens[b])) for b in range(B)])
    assert np.array_equal(Kd.float().cpu().numpy(), lay(want))
    assert list(ld.cpu().numpy()) == [int(lens[b]) + len(paths[b]) for b in range(B)]


def test_commit_without_lengths_and_with_entries_that_are_no_slots():
    import torch
    say("[case] commit: entries that are no slots")
    N, T, d = 6, 10, 16
    K = torch.arange((T + N) * d, device="cuda", dtype=torch.float32).reshape(1, T + N, d)
    before = K.cpu().numpy()[0].copy()
    path = torch.tensor([[0, 99, -4, 1, 5, 7]], dtype=torch.int32, device="cuda")
    new = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.slim_tree_commit(K, path, torch.tensor([50], dtype=torch.int32, device="cuda"), new, 1, N, 2, T, d, dtype="f32")
    torch.cuda.synchronize()
    before[T + 4] = before[T + 5]
    assert np.array_equal(K.cpu().numpy()[0], before) and int(new[0]) == T + N


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("V,dtype", [(300001, "f32"), (1100003, "bf16")])
def test_vocabularies_summed_in_parts_of_parts(V, dtype, draft):
    """Tokens at the vocabulary's very ends, between them, and past a stretch without any weight."""
    say(f"[case] verify: V={V} {dtype} draft={draft}")
    rng = np.random.default_rng(V)
    p, q = _probabilities(rng, 3, 2, V, dtype, draft)
    p[1, :, 1000:V - 5] = 0.0
    parents, tokens = np.tile(np.array([-1, 0], dtype=np.int32), (3, 1)), rng.integers(0, 3, (3, 2)).astype(np.int32)
    for u0 in (0.0, 0.31, 0.77, np.float32(1) - np.float32(2 ** -24)):
        u = np.array([[u0, 0.999]] * 3, dtype=np.float32)
        _same(_call(tokens, parents, p, q if draft else None, u, dtype), tokens, parents, p, q if draft else None, u)
