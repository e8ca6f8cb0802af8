"""Shared plumbing of the tests of drafted trees: seeded caches and trees, and the bound that the result's errors keep.  Not a test module."""
from __future__ import annotations

import numpy as np

from oracle import tree_oracle as orc
from paper_2503_05840_amd import binding, synth

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # half a step of the type, relative


def random_tree(rng, N, used=None, deep=False):
    """Parents of N slots: node 0 a root, every other node below an earlier one (deep: mostly the one before); slots from `used` on are unused."""
    par = [-1] + [i - 1 if deep and rng.random() < 0.8 else int(rng.integers(0, i)) for i in range(1, N)]
    for i in range(used if used is not None else N, N):
        par[i] = -2
    return np.array(par, dtype=np.int32)


class TreeCase:
    """A batch of trees over caches, as arrays that hold exactly what the device holds."""

    def __init__(self, B, N, H, d_k, T, dtype, lens=None, parents=None, base=None, seed=0, q_scale=1.5, banded=False, slack=0):
        rng = np.random.default_rng(seed)
        d = H * d_k
        self.B, self.N, self.H, self.d_k, self.d, self.T, self.dtype, self.base, self.banded = B, N, H, d_k, d, T, dtype, base, banded
        self.rows = T + N + slack
        if banded:
            self.rows = (self.rows + 31) // 32 * 32
        self.lens = np.array([T] * B if lens is None else lens, dtype=np.int32)
        self.given_lens = lens is not None
        self.parents = np.stack([random_tree(rng, N) for _ in range(B)]) if parents is None else np.array(parents, dtype=np.int32).reshape(B, N)
        self.K = synth.round_through(rng.standard_normal((B, self.rows, d)), dtype)
        self.q = synth.round_through(rng.standard_normal((B, N, d)) * q_scale, dtype)
        self.W = synth.round_through(rng.standard_normal((d, d)) / np.sqrt(d), dtype)

    def device(self):
        """The device tensors, made anew from the arrays."""
        import torch
        t = torch.bfloat16 if self.dtype == "bf16" else torch.float32
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(t).contiguous()  # noqa: E731
        K = self.K
        if self.banded:
            K = np.ascontiguousarray(K.reshape(self.B, self.rows // 32, 32, self.H, self.d_k).transpose(0, 1, 3, 2, 4)).reshape(K.shape)
        self.dev = {"q": up(self.q), "K": up(K), "W": up(self.W), "parents": torch.from_numpy(self.parents).cuda(),
                    "lens": torch.from_numpy(self.lens).cuda() if self.given_lens else None,
                    "rope": None if self.base is None else torch.from_numpy(binding.slim_rope_table(self.T + self.N, self.d_k, self.base)).cuda()}
        return self.dev

    def call(self, out=None, **kw):
        import torch
        v = self.dev
        if out is None:
            out = torch.full((self.B, self.N, self.d), float("nan"), dtype=v["q"].dtype, device="cuda")
        kw.setdefault("k_layout", binding.K_BANDED if self.banded else binding.K_ROWMAJOR)
        return binding.slim_tree_decode(v["q"], v["K"], v["W"], v["parents"], out, self.B, self.N, self.H, self.T, self.d, dtype=self.dtype,
                                        seq_lens=v["lens"], t_stride=self.rows, rope_table=v["rope"], **kw)

    def run(self, **kw):
        import torch
        self.device()
        out = self.call(**kw)
        torch.cuda.synchronize()
        return out.float().cpu().numpy()

    def expected(self, sequences=None, nodes=None):
        """(result, bound), both (B, N, d), zeros but for the given sequences and nodes (None: all).  The bound, to first order and then a tenth more for the products of errors:
        a numerator is off by half a step of the type (and the softmax sum is of the rounded ones), by the error of its score and by two steps of
        fp32 for its exponential: spread times that; sums over T rows and d columns in fp32, and C as the type's hi + lo: size times
        that; the result's own rounding."""
        out, bound = np.zeros((self.B, self.N, self.d)), np.zeros((self.B, self.N, self.d))
        f32, half = HALF["f32"], HALF[self.dtype]
        for b in range(self.B) if sequences is None else sequences:
            n = int(self.lens[b])
            o, spread, size, swing = orc.tree_attention(self.q[b], self.K[b, :n + self.N], self.W, self.parents[b], n, self.H, self.base, nodes)
            score = swing * (self.d_k + 4) * f32
            if self.base is not None:
                # angles' cos and sin as fp32, the rotation in fp32, and in bf16 the rotated key as hi + lo
                score = score + swing * 2 * (4 * f32 + (half ** 2 if self.dtype == "bf16" else 0.0))
            delta = (half if self.dtype == "bf16" else 0.0) + 4 * f32 + np.repeat(score, self.d_k, axis=1)
            lo = half ** 2 if self.dtype == "bf16" else 0.0
            bound[b] = 1.1 * (delta * spread + size * ((n + self.N + self.d) * f32 + lo) + half * np.abs(o)) + 1e-30
            out[b] = o
        return out, bound

    def check(self, got=None, **kw):
        got = self.run(**kw) if got is None else got
        want, bound = self.expected()
        assert np.isfinite(got).all()
        worst = np.abs(got - want) / bound
        assert worst.max() <= 1.0, f"{worst.max():.3f} of the bound at {np.unravel_index(worst.argmax(), worst.shape)}"
        return float(worst.max())

    def check_some(self, sequences, nodes, got=None):
        """`check` of a few nodes of a few sequences; the other results have to be finite."""
        got = self.run() if got is None else got
        want, bound = self.expected(sequences, nodes)
        assert np.isfinite(got).all()
        at = np.ix_(sequences, nodes)
        worst = np.abs(got[at] - want[at]) / bound[at]
        assert worst.max() <= 1.0, f"{worst.max():.3f} of the bound at {np.unravel_index(worst.argmax(), worst.shape)}"
        return float(worst.max())
