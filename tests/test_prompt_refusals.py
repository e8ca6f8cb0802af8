"""What the calls for whole prompts and for caches in 4 or 8 bits refuse, on the host and before anything is launched; the oracle's own parts.  CPU only."""
import ctypes

import numpy as np
import pytest

from oracle import prompt_oracle as orc
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


def _swap(n, **at):
    return tuple(at.get(f"p{i}", FAKE) for i in range(n))


def _append(ptrs=_swap(4), B=2, n=8, T=64, d=512, bits=4, pitch=0, o=None):
    return binding.load().slim_quant_append(*ptrs, B, n, T, d, bits, pitch, o if o is not None else _opts())


def _read(ptrs=_swap(4), B=2, n=8, T=64, d=512, bits=4, pitch=0, o=None):
    return binding.load().slim_quant_read(*ptrs, B, n, T, d, bits, pitch, o if o is not None else _opts())


def _decode(ptrs=_swap(5), B=2, H=8, T=64, d=512, bits=4, o=None):
    return binding.load().slim_quant_decode(*ptrs, B, H, T, d, bits, o if o is not None else _opts())


def _prompt(ptrs=_swap(6), B=2, rows_q=40, rows_k=40, H=8, H_kv=2, d_k=64, causal=1, pitches=(0, 0, 0), o=None):
    return binding.load().slim_prompt_attention(*ptrs, B, rows_q, rows_k, H, H_kv, d_k, causal, *pitches, o if o is not None else _opts())


@pytest.mark.parametrize("call,n,optional", [(_append, 4, (1,)), (_read, 4, (2,)), (_decode, 5, ()), (_prompt, 6, (4,))])
def test_null_and_misaligned_pointers(call, n, optional):
    for i in range(n):
        if i not in optional:
            assert call(_swap(n, **{f"p{i}": None})) == ARG, i
        offsets = i in optional or (call is _prompt and i == 3)
        assert call(_swap(n, **{f"p{i}": ODDER if offsets else ODD})) == ALIGN, i


@pytest.mark.parametrize("call", [_append, _read, _decode])
def test_formats_and_rows_of_a_cache(call):
    for bits in (0, 1, 2, 5, 16, -4):
        assert call(bits=bits) == ARG
    assert call(o=_opts(k_layout=1)) == ARG
    for kw in (dict(B=0), dict(B=-1), dict(B=1 << 16), dict(T=0), dict(T=-5), dict(T=(1 << 24) + 1), dict(d=0), dict(d=48), dict(d=520), dict(d=(1 << 20) + 32)):
        assert call(**kw) == SHAPE, kw
    assert call(o=_opts(dtype=4)) == DTYPE
    assert call(o=_opts(t_stride=32)) == SHAPE
    assert call(o=_opts(t_stride=-64)) == SHAPE
    assert call(o=_opts(t_stride=100)) == LAYOUT
    assert call(o=_opts(seq_lens=4098)) == ALIGN
    for bad in ([3, -1], [65, 0]):
        a = np.array(bad, dtype=np.int32)
        assert call(o=_opts(seq_lens_host=a.ctypes.data)) == SEQLEN


@pytest.mark.parametrize("call", [_append, _read])
def test_packed_rows(call):
    plain = dict(p1=None) if call is _append else dict(p2=None)
    assert call(_swap(4, **plain), n=7) == SHAPE               # 7 rows are not as many for each of two sequences
    for n in (-2, (1 << 24) + 2):
        assert call(n=n) == SHAPE
    assert call(n=1 << 24, d=1 << 18, pitch=1 << 18) == SHAPE    # more workgroups than a launch has
    assert call(pitch=-512) == ARG
    for pitch in (511, 504, 516):
        assert call(pitch=pitch) == SHAPE
    assert call(o=_opts(rope_table=4096)) == ARG


def test_decode_heads_and_workspace():
    for kw in (dict(H=0), dict(H=7), dict(H=128), dict(H=2048, d=1 << 14), dict(H=1, d=544)):
        assert _decode(**kw) == SHAPE, kw
    assert _decode(B=32768, H=64, d=2048, o=_opts(t_stride=64)) == SHAPE                     # more groups of heads than a grid has places
    assert _decode(o=_opts(rope_table=4104)) == ALIGN
    need = binding.slim_workspace_bytes_quant(2, 8, 64, 512, 4, "bf16")
    assert need > 0
    assert _decode(o=_opts(workspace=4096, workspace_bytes=need - 1)) == WORKSPACE
    assert _decode(o=_opts(workspace=4104, workspace_bytes=need)) == ALIGN
    assert binding.slim_workspace_bytes_quant(2, 7, 64, 512, 4, "bf16") == 0
    assert binding.slim_workspace_bytes_quant(2, 8, 64, 512, 6, "bf16") == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_workspace_grows_with_the_context(dtype):
    for B, H, d in ((1, 32, 4096), (3, 20, 1280), (16, 24, 2304), (40, 12, 864)):
        last = 0
        for T in sorted({1, 63, 64, 65, 1000, 4096, 5000, 16384, 40000, 131072} | set(range(100, 9000, 137))):
            n = binding.slim_workspace_bytes_quant(B, H, T, d, 4, dtype)
            assert n >= last
            last = n


def test_prompt_shapes_options_and_workspace():
    for kw in (dict(B=0), dict(B=1 << 16), dict(rows_q=-1), dict(rows_k=-1), dict(H=0), dict(H_kv=0), dict(H=6, H_kv=4), dict(d_k=0), dict(d_k=60), dict(d_k=264),
               dict(rows_q=(1 << 24) + 1), dict(H=8192, H_kv=1), dict(H=4096, H_kv=1, rows_q=1 << 20, rows_k=1 << 20)):
        assert _prompt(**kw) == SHAPE, kw
    assert _prompt(_swap(6, p4=None), rows_q=40, rows_k=41) == SHAPE
    assert _prompt(pitches=(-512, 0, 0)) == ARG
    for pitches in (((1 << 24) + 8, 0, 0), (504, 0, 0), (516, 0, 0), (0, 120, 0), (0, 0, 120), (0, 132, 0)):
        assert _prompt(pitches=pitches) == SHAPE, pitches
    assert _prompt(o=_opts(dtype=2)) == DTYPE
    assert _prompt(d_k=36) == SHAPE                              # 16-byte vectors of bf16
    for o in (dict(seq_lens=4096), dict(seq_lens_host=4096), dict(rope_table=4096), dict(k_layout=1), dict(t_stride=64)):
        assert _prompt(o=_opts(**o)) == ARG
    need = binding.slim_workspace_bytes_prompt(1, 1, 8192, 8, 8, 128, "bf16")
    args = dict(B=1, rows_q=1, rows_k=8192, H_kv=8, d_k=128)
    assert _prompt(o=_opts(workspace=4096, workspace_bytes=need - 1), **args) == WORKSPACE
    assert _prompt(o=_opts(workspace=4104, workspace_bytes=need), **args) == ALIGN
    assert binding.slim_workspace_bytes_prompt(1, 1, 8192, 8, 3, 128, "bf16") == 0


def test_binding_checks_shapes_and_types():
    import torch
    t = lambda *s, d=torch.bfloat16: torch.zeros(s, dtype=d)      # noqa: E731  (host tensors: refused for that at the latest)
    i32, u8 = torch.int32, torch.uint8
    with pytest.raises(ValueError):
        binding.slim_quant_append(t(8, 512), t(2, 64, 256, d=u8), t(2, 16, 64, d=u8), 2, 64, 512, 4)
    with pytest.raises(ValueError):
        binding.slim_quant_read(t(2, 64, 256, d=u8), t(2, 16, 64, d=u8), t(8, 511), 2, 64, 512, 4)
    with pytest.raises(ValueError):
        binding.slim_quant_decode(t(2, 512), t(2, 64, 128, d=u8), t(2, 16, 64, d=u8), t(512, 512), t(2, 512), 2, 8, 64, 512, 4)
    with pytest.raises(ValueError):
        binding.slim_prompt_attention(t(40, 512), t(40, 128), t(40, 128), t(3, d=i32), t(40, 512), 2, 8, 2, 64)
    with pytest.raises(ValueError):
        binding.slim_prompt_attention(t(40, 512), t(40, 128), t(40, 128), None, t(40, 512), 2, 8, 2, 64)


@pytest.mark.parametrize("bits", [4, 8])
def test_oracle_format(bits):
    """Every value that the format holds comes back as itself; others go to the nearest one."""
    v = orc.grid(bits)
    assert len(v) == (8 if bits == 4 else 127) and v[-1] == (6 if bits == 4 else 448)
    row = np.zeros(128)
    row[:len(v)] = v
    row[31::32] = v[-1]                                        # (a group's largest value fixes its scale)
    for f in (1.0, -1.0, 2.0 ** 100, 2.0 ** -90):
        codes, scales = orc.quantise(f * row[None], bits)
        assert (orc.values(codes, scales, bits)[0] == f * row).all()
    rng = np.random.default_rng(1)
    x = rng.standard_normal((20, 64)) * np.exp(rng.standard_normal((20, 1)) * 10)
    codes, scales = orc.quantise(x, bits)
    y = orc.values(codes, scales, bits)
    top = np.abs(x).reshape(20, 2, 32).max(-1).repeat(32, -1)
    # Half a step of the binade of the group's largest magnitude: with 4 bits that is 1 of 5 at worst (4 and 6 are neighbours; between 6 and 7, which is
    # cut off, it is 1 of 7), with 8 bits 2^-4.
    assert (np.abs(x - y) <= top * (1 / 5 if bits == 4 else 2.0 ** -4) * 1.0001).all()
    assert (orc.unpack(orc.pack(codes, bits), bits) == codes).all()
    x[3, 40] = np.nan
    x[4, 5] = np.inf
    codes, scales = orc.quantise(x, bits)
    y = orc.values(codes, scales, bits)
    assert np.isnan(y[3, 32:]).all() and np.isfinite(y[3, :32]).all() and np.isnan(y[4, :32]).all() and np.isfinite(y[4, 32:]).all()


def test_oracle_prompt_against_the_vanilla_step():
    from oracle import mha_oracle as vanilla
    rng = np.random.default_rng(2)
    H, d, n = 2, 16, 7
    q, k, v = (rng.standard_normal((n, d)) for _ in range(3))
    out = orc.prompt_attention(q, k, v, H, H, True)[0]
    for i in range(n):
        assert np.allclose(out[i], vanilla.vanilla_decode(q[i], k[:i + 1], v[:i + 1], H), atol=1e-12)
    part = orc.prompt_attention(q[5:], k, v, H, H, True)[0]
    assert np.allclose(part, out[5:], atol=1e-12)
    assert (orc.prompt_attention(q, k[:4], v[:4], H, H, True)[0][:3] == 0).all()
    grouped = orc.prompt_attention(q, k[:, :8], v[:, :8], 2, 1, True)[0]
    assert np.allclose(grouped[:, 8:], orc.prompt_attention(q[:, 8:], k[:, :8], v[:, :8], 1, 1, True)[0], atol=1e-12)
