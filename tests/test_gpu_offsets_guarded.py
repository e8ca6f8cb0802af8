"""Offsets are device data: whatever they are, only rows that there are get read and written, and of these only those that the offsets name.  The buffers lie inside
larger ones whose rest must stay (written) or must not show (read)."""
import numpy as np
import pytest

from oracle import prompt_oracle as orc
from paper_2503_05840_amd import binding
from prompt_cases import PromptCase, ints

pytestmark = pytest.mark.gpu

GUARD = 1 << 16


def _inside(a, fill):
    """A copy of a device tensor in the middle of a larger buffer: (copy, the buffers before and behind)."""
    import torch
    wide = torch.full((2 * GUARD + a.numel(),), fill, dtype=a.dtype, device="cuda")
    mine = wide[GUARD:GUARD + a.numel()].view(a.shape)
    mine.copy_(a)
    return mine, (wide[:GUARD], wide[GUARD + a.numel():])


def _named(cu, n):
    """Packed row -> places (sequence, row of that sequence) that the offsets name for it."""
    return {r: {(b, r - cu[b]) for b in range(len(cu) - 1) if cu[b] <= r < cu[b + 1]} for r in range(n)}


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("start", [None, [120, 90], [-3, 1 << 30], [5, (1 << 31) - 1]])
def test_rows_of_a_cache(bits, dtype, start):
    import torch
    rng = np.random.default_rng(bits)
    B, n, d, T, stride = 2, 20, 96, 125, 192
    held = [0, 0] if start is None else start
    rows = torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    want_c, want_s = orc.quantise(rows.double().cpu().numpy(), bits)
    want_c = orc.pack(want_c, bits)
    rows, _ = _inside(rows, float("nan"))
    kw = dict(dtype=dtype, t_stride=stride, seq_lens=None if start is None else ints(start))
    for cu in ([0, 9, 20], [0, 9, 5000], [-4, 9, 20], [15, 3, 20], [20, 20, 20], [5, 12, 17], [0, 0, 20], [1 << 30, 0, -1], [-(1 << 31), -(1 << 31), 7]):
        c0 = torch.from_numpy(rng.integers(0, 256, (B, stride, d * bits // 8), dtype=np.uint8)).cuda()
        s0 = torch.from_numpy(rng.integers(0, 255, (B, d // 32, stride), dtype=np.uint8)).cuda()
        codes, codes_guard = _inside(c0, 0xa5)
        scales, scales_guard = _inside(s0, 0xa5)
        out, out_guard = _inside(torch.full_like(rows, 77.0), 55.0)
        binding.slim_quant_append(rows, codes, scales, B, T, d, bits, cu_rows=ints(cu), **kw)
        torch.cuda.synchronize()
        named = _named(cu, n)
        changed = (codes != c0).any(-1) | (scales != s0).any(1)
        at = {}
        for r, places in named.items():
            for b, t in places:
                if 0 <= held[b] + t < T:
                    at.setdefault((b, held[b] + t), set()).add(r)
        for b, t in changed.nonzero().tolist():
            assert any((codes[b, t].cpu().numpy() == want_c[r]).all() and (scales[b, :, t].cpu().numpy() == want_s[r]).all() for r in at.get((b, t), ())), (cu, b, t)
        if all(x <= y for x, y in zip(cu, cu[1:])):                # (increasing: every row that has a place is there)
            for (b, t), who in at.items():
                assert all((codes[b, t].cpu().numpy() == want_c[r]).all() for r in who), (cu, b, t)
        binding.slim_quant_read(codes, scales, out, B, T, d, bits, cu_rows=ints(cu), **kw)
        torch.cuda.synchronize()
        assert all((g == 0xa5).all() for g in (*codes_guard, *scales_guard)) and all((g == 55.0).all() for g in out_guard), cu
        touched = (out != 77.0).any(-1).tolist()
        assert not any(touched[r] and not named[r] for r in range(n)), cu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,heads", [(100, 2), (20, 1)])
def test_rows_of_a_prompt(dtype, causal, n, heads):
    """Keys beside the buffer are NaN, and so would be a query that saw them."""
    import torch
    n_k = 100 if n == 100 else 3000                              # (few queries: the keys are cut)
    c = PromptCase([n], [n_k], heads, heads, 64, dtype, causal, seed=6)
    c.device()
    for name in ("q", "k", "v"):
        c.dev[name], _ = _inside(c.dev[name], float("nan"))
    clean = torch.full((n, heads * 64), 77.0, dtype=c.dev["q"].dtype, device="cuda")
    far = 1 << 30
    cu_ks = [None] if n_k == n else [[0, n_k // 2, n_k], [0, n_k, 5 * n_k], [-9, n_k, n_k], [n_k, 10, far], [far, far, far], [0, 0, far]]
    for cu_q in ([0, n // 2, n], [0, n // 2, 50 * n], [-7, n // 2, n], [n - 1, n // 5, n], [n, 0, 0], [far, far, far], [-far, -far, far], [0, far, far]):
        for cu_k in cu_ks:
            out, guard = _inside(clean, 55.0)
            binding.slim_prompt_attention(c.dev["q"], c.dev["k"], c.dev["v"], ints(cu_q), out, 2, heads, heads, 64, cu_k=None if cu_k is None else ints(cu_k),
                                          causal=causal, dtype=dtype)
            torch.cuda.synchronize()
            assert all((g == 55.0).all() for g in guard), (cu_q, cu_k)
            named = _named(cu_q, n)
            touched = (out != 77.0).any(-1).tolist()
            assert not any(touched[r] and not named[r] for r in range(n)), (cu_q, cu_k)
            if all(x <= y for x, y in zip(cu_q, cu_q[1:])):
                assert all(touched[r] for r in range(n) if named[r]) and torch.isfinite(out).all(), (cu_q, cu_k)
