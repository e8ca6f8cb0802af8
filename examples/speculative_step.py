"""Speculative decoding with trees of drafted tokens, on a model of one attention layer with random weights: every step checks N drafted tokens of each
sequence at once (slim_tree_decode), accepts those that the model itself would have taken (slim_tree_verify) and keeps their keys (slim_tree_commit).

    python examples/speculative_step.py [steps]

The model decodes greedily: its probabilities are one-hot, so the tokens are exactly those of one step after the other (`one_by_one`).  The
lengths stay on the device; nothing in the loop waits for the GPU.
"""
from __future__ import annotations

import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2503_05840_amd import binding  # noqa: E402

PARENTS = [-1, 0, 0, 1, 1, 2, 2, 3]        # the last token, two guesses for the next, two for each of theirs, one deeper


class Model:
    """Embedding, one attention layer over a K-cache, vocabulary.  The draft guesses what would follow a token if nothing stood before it."""

    def __init__(self, V=512, H=8, d=512, seed=0):
        import torch
        rng = np.random.default_rng(seed)
        up = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()  # noqa: E731
        self.V, self.H, self.d = V, H, d
        W_K = np.linalg.qr(rng.standard_normal((d, d)))[0]   # (far from singular: W_KV = W_K^-1 W_V exists and is small)
        W_V = rng.standard_normal((d, d)) / np.sqrt(d)
        W_KV, _ = binding.slim_prepare_wkv(W_K, W_V)
        self.emb, self.W_Q, self.W_K = up(rng.standard_normal((V, d))), up(rng.standard_normal((d, d)) / np.sqrt(d)), up(W_K)
        self.W_KV, self.head = up(W_KV), up(rng.standard_normal((d, V)) / np.sqrt(d))
        self.guesses = self.logits(self.emb, self.emb @ up(W_V)).topk(2, -1).indices.to(torch.int32)

    def logits(self, x, attention):
        return (x + attention) @ self.head

    def greedy(self, x, attention):
        """The distribution of a greedy model: all of it on the likeliest token."""
        import torch
        logits = self.logits(x, attention)
        return torch.zeros_like(logits).scatter_(-1, logits.argmax(-1, keepdim=True), 1.0)


def tree_of(model, last, parents):
    """Tokens (B, N) of the tree below the last tokens (B,): a node's children are the guesses for it, the likelier first."""
    import torch
    tokens = [last]
    for i, up in enumerate(parents[1:], 1):
        tokens.append(model.guesses[tokens[up].long(), parents[1:i].count(up)])
    return torch.stack(tokens, 1).contiguous()


def speculative(model, prompt_keys, lens, last, steps, parents=None):
    """prompt_keys (B, T, d), lens (B,), last (B,): `steps` steps.  Returns per sequence the tokens after `last`."""
    import torch
    parents = parents or PARENTS
    B, T, d = prompt_keys.shape
    N, H = len(parents), model.H
    room = T + steps * N                                 # every step may keep all its nodes
    K = torch.zeros((B, room + N, d), device="cuda")
    K[:, :T] = prompt_keys
    lens, b = lens.clone(), torch.arange(B, device="cuda")[:, None]
    par = torch.tensor([parents] * B, dtype=torch.int32, device="cuda")
    u = torch.full((B, N), 0.5, device="cuda")           # (a one-hot distribution leaves nothing to chance)
    out = torch.empty((B, N, d), device="cuda")
    ws = torch.empty(binding.slim_workspace_bytes_tree(B, N, H, room, d, "f32"), dtype=torch.uint8, device="cuda")
    made = []
    for _ in range(steps):
        tokens = tree_of(model, last, parents)
        x = model.emb[tokens.long()]
        K[b, lens[:, None] + torch.arange(N, device="cuda")] = x @ model.W_K
        binding.slim_tree_decode(x @ model.W_Q, K, model.W_KV, par, out, B, N, H, room, d, dtype="f32", seq_lens=lens, workspace=ws)
        p = model.greedy(x, out)
        path, n_path, last = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((B, N), (B,), (B,)))
        binding.slim_tree_verify(tokens, par, p, None, u, path, n_path, last, B, N, model.V)
        binding.slim_tree_commit(K, path, n_path, lens, B, N, H, room, d, dtype="f32", seq_lens=lens)
        made.append((tokens, path, n_path, last))
    result = [[] for _ in range(B)]
    for tokens, path, n_path, nxt in made:
        tokens, path, n_path, nxt = (t.cpu().tolist() for t in (tokens, path, n_path, nxt))
        for i in range(B):
            result[i] += [tokens[i][j] for j in path[i][1:n_path[i]]] + [nxt[i]]
    return result


def one_by_one(model, prompt_keys, lens, last, count):
    """The same model, one token a step (slim_decode): `count` tokens of every sequence."""
    import torch
    B, T, d = prompt_keys.shape
    K = torch.zeros((B, T + count, d), device="cuda")
    K[:, :T] = prompt_keys
    lens, b = lens.clone(), torch.arange(B, device="cuda")
    out, result = torch.empty((B, d), device="cuda"), []
    for _ in range(count):
        x = model.emb[last.long()]
        K[b, lens.long()] = x @ model.W_K
        lens += 1
        binding.slim_decode(x @ model.W_Q, K, model.W_KV, out, B, model.H, T + count, d, dtype="f32", seq_lens=lens)
        last = model.logits(x, out).argmax(-1).to(torch.int32)
        result.append(last)
    return torch.stack(result, 1).cpu().tolist()


def prompts(model, B=4, T=300, seed=1):
    """Keys of random prompts of several lengths, and their last tokens (whose keys the first step makes)."""
    import torch
    rng = np.random.default_rng(seed)
    tokens = torch.from_numpy(rng.integers(0, model.V, (B, T))).cuda()
    lens = torch.tensor([T - 37 * i for i in range(B)], dtype=torch.int32, device="cuda")
    last = torch.from_numpy(rng.integers(0, model.V, B).astype(np.int32)).cuda()
    return model.emb[tokens] @ model.W_K, lens, last


def main():
    steps = int(sys.argv[1]) if len(sys.argv) > 1 else 24
    model = Model()
    keys, lens, last = prompts(model)
    got = speculative(model, keys, lens, last, steps)
    want = one_by_one(model, keys, lens, last, max(len(t) for t in got))
    for i, tokens in enumerate(got):
        print(f"sequence {i}: {len(tokens)} tokens in {steps} steps ({len(tokens) / steps:.2f} a step), "
              f"{'as' if tokens == want[i][:len(tokens)] else 'NOT as'} one by one")


if __name__ == "__main__":
    main()
