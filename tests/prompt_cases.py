"""Shared plumbing of the tests of whole prompts and of caches in 4 or 8 bits: seeded inputs and the bounds that the results' errors keep.  Not a test module."""
from __future__ import annotations

import numpy as np

from oracle import prompt_oracle as orc
from oracle import tree_oracle
from paper_2503_05840_amd import binding, synth

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # half a step of the type, relative
F32 = HALF["f32"]


def up(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32).contiguous()


def ints(a):
    import torch
    return torch.tensor([int(x) for x in a], dtype=torch.int32, device="cuda")


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)])


class PromptCase:
    """Packed sequences of n_q queries and n_k keys each, as arrays that hold exactly what the device holds; `tail` rows of no sequence behind them."""

    def __init__(self, n_q, n_k, H, H_kv, d_k, dtype="bf16", causal=True, seed=0, q_scale=1.5, tail=0):
        rng = np.random.default_rng(seed)
        self.n_q, self.n_k, self.H, self.H_kv, self.d_k, self.dtype, self.causal, self.tail = list(n_q), list(n_k), H, H_kv, d_k, dtype, causal, tail
        self.own_keys = self.n_q != self.n_k
        draw = lambda n, w, s: synth.round_through(rng.standard_normal((n, w)) * s, dtype)  # noqa: E731
        self.q = draw(sum(n_q) + tail, H * d_k, q_scale)
        self.k = draw(sum(n_k) + tail, H_kv * d_k, 1.0)
        self.v = draw(sum(n_k) + tail, H_kv * d_k, 1.0)

    def device(self):
        self.dev = {"q": up(self.q, self.dtype), "k": up(self.k, self.dtype), "v": up(self.v, self.dtype), "cu_q": ints(offsets(self.n_q)),
                    "cu_k": ints(offsets(self.n_k)) if self.own_keys else None}
        return self.dev

    def call(self, out=None, **kw):
        import torch
        x = self.dev
        if out is None:
            out = torch.full((x["q"].shape[0], self.H * self.d_k), 77.0, dtype=x["q"].dtype, device="cuda")
        return binding.slim_prompt_attention(x["q"], x["k"], x["v"], x["cu_q"], out, len(self.n_q), self.H, self.H_kv, self.d_k, cu_k=x["cu_k"],
                                             causal=self.causal, dtype=self.dtype, **kw)

    def run(self, **kw):
        import torch
        self.device()
        out = self.call(**kw)
        torch.cuda.synchronize()
        return out.float().cpu().numpy().astype(np.float64)

    def expected(self, sequence, queries=None):
        """(result, bound) of one sequence.  The bound, to first order and a tenth more: a numerator is off by half a step of the type where it enters the product, the
        sum is of what it was before (so that the error counts against the size, not the spread), scores by their fp32 products and sums, exponentials by four
        steps of fp32; sums over the keys in fp32, and the result's own rounding."""
        q0, k0 = offsets(self.n_q)[sequence], offsets(self.n_k)[sequence]
        n_k = self.n_k[sequence]
        o, spread, size, swing = orc.prompt_attention(self.q[q0:q0 + self.n_q[sequence]], self.k[k0:k0 + n_k], self.v[k0:k0 + n_k], self.H, self.H_kv,
                                                      self.causal, queries)
        score = np.repeat(swing * (self.d_k + 8) * F32, self.d_k, axis=1)
        half = HALF[self.dtype]
        numer = half if self.dtype == "bf16" else 0.0
        bound = 1.1 * ((4 * F32 + score) * spread + size * (numer + (n_k + 4) * F32) + half * np.abs(o)) + 1e-30
        return o, bound

    def check(self, got=None, sequences=None, queries=None, **kw):
        got = self.run(**kw) if got is None else got
        at = offsets(self.n_q)
        worst = 0.0
        for b in range(len(self.n_q)) if sequences is None else sequences:
            want, bound = self.expected(b, queries)
            mine = got[at[b]:at[b + 1]]
            if queries is not None:
                mine, want, bound = mine[queries], want[queries], bound[queries]
            if mine.size:
                assert np.isfinite(mine).all(), f"sequence {b}"
                r = np.abs(mine - want) / bound
                assert r.max() <= 1.0, f"sequence {b}: {r.max():.3f} of the bound at {np.unravel_index(r.argmax(), r.shape)}"
                worst = max(worst, float(r.max()))
        assert (got[at[-1]:] == 77.0).all(), "rows of no sequence were written"
        return worst


class QuantCase:
    """Caches in 4 or 8 bits whose rows behind a sequence's length hold anything (scales that stand for NaN, codes of NaN)."""

    def __init__(self, B, H, d_k, T, bits, dtype="bf16", lens=None, base=None, seed=0, q_scale=1.2, slack=0):
        rng = np.random.default_rng(seed)
        d = H * d_k
        self.B, self.H, self.d_k, self.d, self.T, self.bits, self.dtype, self.base = B, H, d_k, d, T, bits, dtype, base
        self.rows = (T + slack + 63) // 64 * 64
        self.lens = np.array([T] * B if lens is None else lens)
        self.given_lens = lens is not None
        self.codes = rng.integers(0, 256, size=(B, self.rows, d * bits // 8), dtype=np.uint8)
        self.scales = rng.integers(250, 256, size=(B, d // 32, self.rows), dtype=np.uint8)
        self.K = []
        for b in range(B):
            n = int(self.lens[b])
            # codes drawn at once (a rounding of rows is the append's business), scales of unit rows with a few wider groups
            one = rng.integers(0, 16 if bits == 4 else 256, size=(n, d), dtype=np.uint8)
            if bits == 8:
                one = np.where(one & 127 > 0x7c, one ^ 8, one).astype(np.uint8)
            sc = rng.integers(124, 128, size=(n, d // 32)).astype(np.uint8) - (0 if bits == 4 else 6)
            self.codes[b, :n] = orc.pack(one, bits)
            self.scales[b, :, :n] = sc.T
            self.K.append(orc.values(one, sc, bits))
        self.q = synth.round_through(rng.standard_normal((B, d)) * q_scale, dtype)
        self.W = synth.round_through(rng.standard_normal((d, d)) / np.sqrt(d), dtype)

    def device(self):
        import torch
        self.dev = {"q": up(self.q, self.dtype), "W": up(self.W, self.dtype), "codes": torch.from_numpy(self.codes).cuda(),
                    "scales": torch.from_numpy(self.scales).cuda(), "lens": ints(self.lens) if self.given_lens else None,
                    "rope": None if self.base is None else torch.from_numpy(binding.slim_rope_table(self.T, self.d_k, self.base)).cuda()}
        return self.dev

    def call(self, out=None, **kw):
        import torch
        x = self.dev
        if out is None:
            out = torch.full((self.B, self.d), float("nan"), dtype=x["q"].dtype, device="cuda")
        return binding.slim_quant_decode(x["q"], x["codes"], x["scales"], x["W"], out, self.B, self.H, self.T, self.d, self.bits, dtype=self.dtype,
                                         seq_lens=x["lens"], t_stride=self.rows, rope_table=x["rope"], **kw)

    def run(self, **kw):
        import torch
        self.device()
        out = self.call(**kw)
        torch.cuda.synchronize()
        return out.float().cpu().numpy().astype(np.float64)

    def expected(self, b):
        """(result, bound) of one sequence; the bound as for a drafted token: half a step of the type for a numerator (the sum is of the rounded ones), fp32
        scores, exponentials, sums over rows and columns, the weighted sum as hi + lo of the type, and the result's own rounding."""
        n = int(self.lens[b])
        if n == 0:
            return np.zeros(self.d), np.full(self.d, 1e-30)
        o, spread, size, swing = (x[0] for x in tree_oracle.tree_attention(self.q[b:b + 1], self.K[b], self.W, [-1], n - 1, self.H, self.base))
        half = HALF[self.dtype]
        score = np.repeat(swing * (self.d_k + 8 + (0 if self.base is None else 12)) * F32, self.d_k)
        delta = (half if self.dtype == "bf16" else 0.0) + 4 * F32 + score
        lo = half ** 2 if self.dtype == "bf16" else 0.0
        return o, 1.1 * (delta * spread + size * ((n + self.d) * F32 + lo) + half * np.abs(o)) + 1e-30

    def check(self, got=None, sequences=None, **kw):
        got = self.run(**kw) if got is None else got
        assert np.isfinite(got).all()
        worst = 0.0
        for b in range(self.B) if sequences is None else sequences:
            want, bound = self.expected(b)
            r = np.abs(got[b] - want) / bound
            assert r.max() <= 1.0, f"sequence {b}: {r.max():.3f} of the bound at column {r.argmax()}"
            worst = max(worst, float(r.max()))
        return worst
