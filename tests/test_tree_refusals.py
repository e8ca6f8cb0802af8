"""What the calls for drafted trees refuse, on the host and before anything is launched; the oracle's own parts.  CPU only."""
import ctypes

import numpy as np
import pytest

from oracle import tree_oracle as orc
from paper_2503_05840_amd import binding

FAKE = ctypes.c_void_p(4096)          # never dereferenced: validation fails first
ODD = ctypes.c_void_p(4104)
ODDER = ctypes.c_void_p(4098)
ARG, SHAPE, DTYPE, ALIGN, WORKSPACE, SEQLEN, LAYOUT = -1, -2, -3, -4, -5, -9, -11


def _opts(**kw):
    o = binding.SlimOpts()
    o.dtype = binding.SLIM_BF16
    for k, v in kw.items():
        setattr(o, k, v)
    return ctypes.byref(o)


def _decode(ptrs=(FAKE,) * 5, B=1, N=4, H=8, T=16, d=512, o=None):
    return binding.load().slim_tree_decode(*ptrs, B, N, H, T, d, o if o is not None else _opts())


def _commit(ptrs=(FAKE,) * 4, B=1, N=4, H=8, T=16, d=512, o=None):
    return binding.load().slim_tree_commit(*ptrs, B, N, H, T, d, o if o is not None else _opts())


def _verify(ptrs=(FAKE,) * 8, B=1, N=4, V=100, o=None):
    return binding.load().slim_tree_verify(*ptrs, B, N, V, o if o is not None else _opts())


@pytest.mark.parametrize("call,n", [(_decode, 5), (_commit, 4), (_verify, 8)])
def test_null_pointers(call, n):
    for i in range(n):
        if call is _verify and i == 3:
            continue                                              # (no distribution of the draft: allowed)
        assert call(tuple(None if k == i else FAKE for k in range(n))) == ARG


@pytest.mark.parametrize("call", [_decode, _commit])
def test_shapes_types_and_layouts_of_the_cache(call):
    for kw in (dict(B=0), dict(B=1 << 16), dict(N=0), dict(N=65), dict(H=0), dict(H=7), dict(T=-1), dict(T=1 << 24), dict(d=0), dict(H=128),
               dict(H=1, d=(1 << 20) + 8), dict(N=-3), dict(B=-1)):
        assert call(**kw) == SHAPE, kw
    assert call(o=_opts(t_stride=19)) == SHAPE                    # T + N rows are needed
    assert call(o=_opts(t_stride=-4)) == SHAPE
    assert call(o=_opts(dtype=7)) == DTYPE
    assert call(o=_opts(k_layout=2)) == ARG
    assert call(o=_opts(k_layout=1)) == LAYOUT                    # T + N = 20 rows
    assert call(o=_opts(k_layout=1, t_stride=40)) == LAYOUT
    assert call(o=_opts(seq_lens=4098)) == ALIGN


@pytest.mark.parametrize("call", [_decode, _commit])
def test_host_lengths(call):
    for lens, rc in (([16, -1], SEQLEN), ([17, 3], SEQLEN)):
        a = np.array(lens, dtype=np.int32)
        assert call(B=2, o=_opts(seq_lens_host=a.ctypes.data)) == rc


def test_alignment_rope_and_workspace():
    for i in (0, 1, 2, 4):
        assert _decode(tuple(ODD if k == i else FAKE for k in range(5))) == ALIGN
    assert _decode((FAKE, FAKE, FAKE, ODDER, FAKE)) == ALIGN
    assert _decode(o=_opts(rope_table=4104)) == ALIGN
    assert _decode(o=_opts(workspace=4096, workspace_bytes=64)) == WORKSPACE
    need = binding.slim_workspace_bytes_tree(1, 4, 8, 16, 512, "bf16")
    assert _decode(o=_opts(workspace=4096, workspace_bytes=need - 1)) == WORKSPACE
    assert _decode(o=_opts(workspace=4104, workspace_bytes=need)) == ALIGN
    assert _commit(o=_opts(rope_table=4096)) == ARG
    assert _commit((ODD, FAKE, FAKE, FAKE)) == ALIGN
    for i in (1, 2, 3):
        assert _commit(tuple(ODDER if k == i else FAKE for k in range(4))) == ALIGN


def test_verification():
    for kw in (dict(B=0), dict(N=0), dict(N=65), dict(V=0), dict(V=(1 << 24) + 1), dict(B=1 << 16)):
        assert _verify(**kw) == SHAPE, kw
    assert _verify(o=_opts(dtype=3)) == DTYPE
    for o in (dict(seq_lens=4096), dict(rope_table=4096), dict(k_layout=1), dict(t_stride=8)):
        assert _verify(o=_opts(**o)) == ARG
    for i in range(8):
        ptr = ODD if i in (2, 3) else ODDER
        assert _verify(tuple(ptr if k == i else FAKE for k in range(8))) == ALIGN


def test_workspace_grows_with_every_size_and_refuses_what_the_call_refuses():
    size = lambda *a: binding.slim_workspace_bytes_tree(*a, "bf16")  # noqa: E731
    assert size(1, 65, 8, 16, 512) == 0 and size(1, 4, 7, 16, 512) == 0 and size(0, 4, 8, 16, 512) == 0
    for B, N, H, d in ((1, 1, 8, 512), (3, 7, 20, 1280), (8, 64, 32, 4096), (2, 33, 12, 864)):
        last = 0
        for T in sorted({0, 1, 100, 255, 256, 257, 1000, 1023, 1024, 4000, 4096, 5000, 16384, 40000} | set(range(190, 2300, 31))):
            n = size(B, N, H, T, d)
            assert n >= last
            last = n


def test_binding_checks_shapes_and_types():
    import torch
    t = lambda *s, d=torch.bfloat16: torch.zeros(s, dtype=d)      # noqa: E731  (host tensors: the shape is looked at first)
    i32 = torch.int32
    with pytest.raises(ValueError):
        binding.slim_tree_decode(t(1, 3, 64), t(1, 20, 64), t(64, 64), t(1, 4, d=i32), t(1, 4, 64), 1, 4, 1, 16, 64)
    with pytest.raises(ValueError):
        binding.slim_tree_verify(t(1, 4, d=torch.int64), t(1, 4, d=i32), t(1, 4, 9), None, t(1, 4), t(1, 4, d=i32), t(1, d=i32), t(1, d=i32), 1, 4, 9)
    with pytest.raises(ValueError):
        binding.slim_tree_commit(t(1, 19, 64), t(1, 4, d=i32), t(1, d=i32), t(1, d=i32), 1, 4, 1, 16, 64)


def test_oracle_tree_attention_against_the_vanilla_step_and_by_hand():
    from oracle import mha_oracle as vanilla
    rng = np.random.default_rng(3)
    H, d, T, N = 2, 16, 9, 5
    K, W, q = rng.standard_normal((T + N, d)), rng.standard_normal((d, d)), rng.standard_normal((N, d))
    out = orc.tree_attention(q, K, W, [-1, 0, 1, 2, 3], T, H)[0]
    for i in range(N):
        n = T + i + 1
        assert np.allclose(out[i], vanilla.vanilla_decode(q[i], K[:n], K[:n] @ W, H), atol=1e-12)
    assert orc.chain([-1, 0, 1, 9, 3], 4) is None and orc.chain([-1, 0, 0, 2], 3) == [3, 2, 0]


def test_oracle_verification_gives_the_target_distribution():
    """Accepted tokens and the one after, over many draws: the first token after the root is distributed as the target's, drawn or chosen."""
    rng = np.random.default_rng(4)
    V, N, n = 5, 4, 20000
    p = rng.dirichlet(np.ones(V), size=N)
    q = rng.dirichlet(np.ones(V), size=N)
    for drawn in (True, False):
        seen = np.zeros(V)
        for _ in range(n):
            tokens = [0] + list(rng.choice(V, size=3, p=q[0])) if drawn else [0, 1, 3, 1]
            path, nxt = orc.verify(tokens, [-1, 0, 0, 0], p, q if drawn else None, rng.random(N))
            seen[tokens[path[1]] if len(path) > 1 else nxt] += 1
        # five standard deviations of a count of n draws
        assert np.abs(seen / n - p[0]).max() <= 5 * 0.5 / np.sqrt(n)
