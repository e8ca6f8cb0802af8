"""The calls that a step of speculative decoding makes of this library, and the same in plain torch: attention of a tree of
drafted tokens over a K-cache, verification of the tree against the target's probabilities, and the commit of the accepted
path to the cache.

A case is a plain dict.  `op` says which operator; the other entries:
  tree    B, N (drafted tokens a sequence), H, d_k, T (rows of context that the cache holds), lo (0: every sequence has T rows of context; else the
          lengths spread from lo to T), dtype ("bf16" | "f32": cache, weights, queries and result), rope (keys carry rotary positions), banded (the
          cache's layout), used (nodes of the smallest tree of the batch; the others have up to N)
  verify  B, N, V (vocabulary), dtype of the probabilities, draft (the children were drawn from a distribution that is given; else chosen)
  commit  B, N, H, d_k, T, lo, dtype, banded

Values are random, on the scale that a trained layer has them: unit keys, weights of variance 1 / fan-in, queries whose scores spread by one
or two; vocabularies' probabilities are softmax rows of logits that spread by three, the draft's logits are the target's with noise.
"""
import math

import torch

own = False

_T = {"bf16": torch.bfloat16, "f32": torch.float32}


def _tree(name, B, N, H, d_k, T, lo=0, dtype="bf16", rope=False, banded=False, used=0):
    return {"name": name, "op": "tree", "B": B, "N": N, "H": H, "d_k": d_k, "T": T, "lo": lo, "dtype": dtype, "rope": rope,
            "banded": banded, "used": used or N}


def _verify(name, B, N, V, dtype="f32", draft=True):
    return {"name": name, "op": "verify", "B": B, "N": N, "V": V, "dtype": dtype, "draft": draft}


def _commit(name, B, N, H, d_k, T, lo=0, dtype="bf16", banded=False):
    return {"name": name, "op": "commit", "B": B, "N": N, "H": H, "d_k": d_k, "T": T, "lo": lo, "dtype": dtype, "banded": banded}


def listed():
    return [
        # a full-precision cache in a small ragged batch, small trees: a model served as it was trained
        _tree("tree f32 batch", 4, 13, 16, 64, 1500, lo=300, dtype="f32", used=9),
        # one token of one sequence on a 7B-shaped layer: the tree that has only its root
        _tree("tree one token", 1, 1, 32, 128, 777),
        # one chat turn on the same layer: short odd context, a few drafted tokens; latency and launches
        _tree("tree short", 1, 7, 32, 128, 777),
        # the same layer at its full context, a middling tree
        _tree("tree 16k", 1, 26, 32, 128, 16384),
        # rotary keys, ragged contexts of a chat batch, trees of several sizes
        _tree("tree rotary ragged", 8, 16, 24, 96, 5000, lo=600, rope=True, used=10),
        # narrow heads, a batch in the banded layout
        _tree("tree banded", 16, 21, 20, 64, 1504, lo=500, banded=True),
        # the largest: a batch of full trees over a long context
        _tree("tree full batch", 8, 64, 32, 128, 4096),
        # one sequence's tree against a vocabulary: latency
        _verify("verify one", 1, 8, 32000),
        # a batch, an odd vocabulary, probabilities as a model in bf16 writes them
        _verify("verify batch bf16", 32, 16, 50257, dtype="bf16"),
        # chosen drafts (no distribution of theirs) over a large vocabulary
        _verify("verify chosen large", 8, 26, 128000, draft=False),
        # the accepted path of one sequence, and of a full batch in the banded layout
        _commit("commit one", 1, 8, 32, 128, 2048),
        _commit("commit batch banded", 64, 64, 20, 64, 1504, lo=300, banded=True),
    ]


def _lens(c):
    """Rows of context of every sequence: T, or spread over lo..T in a fixed order that is neither sorted nor periodic."""
    B, T, lo = c["B"], c["T"], c["lo"]
    if not lo:
        return [T] * B
    return [T] + [lo + int((T - lo) * (b * 0.6180339887498949 % 1.0)) for b in range(1, B)]


def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def work(case):
    """tree: K, W_KV, q and the result once; scores, sums and projection of every node as if all were used.  verify: at least the two rows
    (one without a distribution of the draft) that the next token is drawn from.  commit: what a path of a quarter of the nodes moves."""
    c = case
    B, N, z = c["B"], c["N"], _esize(c)
    if c["op"] == "verify":
        rows = 2 if c["draft"] else 1
        return {"bytes": B * (rows * c["V"] * z + 16 * N), "flops": 0}
    d = c["H"] * c["d_k"]
    if c["op"] == "commit":
        return {"bytes": 2 * B * max(1, N // 4) * d * z, "flops": 0}
    n = sum(_lens(c)) + B * N
    return {"bytes": n * d * z + d * d * z + 2 * B * N * d * z + 4 * B * N,
            "flops": 2 * n * N * d + 2 * n * N * c["H"] * d + 2 * B * N * d * d}


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 4e12, w["flops"] / 5e14)


def draw(rng):
    """One more call from the same ranges: a listed kind with other sizes, odd ones among them."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["tree", "tree", "tree", "tree f32", "verify", "verify", "commit"])
        if kind == "verify":
            c = _verify("", spread(1, 64), spread(1, 64), spread(1000, 130000), rng.choice(["f32", "bf16"]), rng.random() < 0.7)
            if c["B"] * c["N"] * c["V"] > 64 << 20:
                continue
        elif kind == "commit":
            H, d_k = rng.choice([(32, 128), (24, 96), (20, 64), (12, 80)])
            banded = rng.random() < 0.5
            T = spread(50, 4000)
            T = (T + 31) // 32 * 32 if banded else T
            c = _commit("", spread(1, 64), spread(1, 64), H, d_k, T, lo=rng.choice([0, max(1, T // 5)]), dtype="bf16" if banded else rng.choice(["bf16", "f32"]), banded=banded)
            if c["B"] * c["T"] * H * d_k > 1 << 29:
                continue
        elif kind == "tree f32":
            N, T = spread(1, 40), spread(40, 3000)
            c = _tree("", spread(1, 8), N, rng.choice([4, 8, 12, 16]), 64, T, lo=rng.choice([0, max(1, T // 5)]), dtype="f32",
                      rope=rng.random() < 0.3, used=rng.randint(1, N))
        else:
            H, d_k = rng.choice([(32, 128), (24, 96), (20, 64), (32, 80), (16, 128), (40, 128), (12, 72)])
            N, T = spread(1, 64), spread(60, 20000)
            banded = H <= 32 and rng.random() < 0.3
            T = (T + 31) // 32 * 32 if banded else T
            c = _tree("", spread(1, 24), N, H, d_k, T, lo=rng.choice([0, max(1, T // 6)]), rope=rng.random() < 0.3, banded=banded,
                      used=rng.randint(max(1, N // 2), N))
            if c["B"] * (T + N) * H * d_k > 3 << 28:
                continue
        if _cost(c) <= most:
            return {k: v for k, v in c.items() if k != "name"}


# ---- inputs -------------------------------------------------------------------------------------------

def _banded(K, H):
    """[B][rows][d], whole bands of 32 rows: head-major inside a band, as the library's banded layout has it."""
    B, rows, d = K.shape
    return K.view(B, rows // 32, 32, H, d // H).transpose(2, 3).contiguous().view(B, rows, d)


def _unbanded(K, H):
    B, rows, d = K.shape
    return K.view(B, rows // 32, H, 32, d // H).transpose(2, 3).contiguous().view(B, rows, d)


def _stride(c):
    rows = c["T"] + c["N"]
    return (rows + 31) // 32 * 32 if c["banded"] else rows


def _parents(c, g):
    """Trees as a drafting model grows them: node 0 is the root, a node's parent is one of the nodes shortly before it."""
    B, N = c["B"], c["N"]
    r = torch.rand((B, N), generator=g, device="cuda")
    i = torch.arange(N, device="cuda").expand(B, N)
    par = (i.float() * (0.3 + 0.7 * r)).long().clamp(max=N)
    par = torch.minimum(par, i - 1)                      # (node 0: -1)
    if c.get("used", N) < N:                             # the trees of a batch have from `used` to N nodes; the slots behind are unused
        n = c["used"] + (torch.arange(B, device="cuda") * 7) % (N - c["used"] + 1)
        par = torch.where(i < n[:, None], par, torch.full_like(par, -2))
    return par.to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"c": c, "own": None}
    B, N = c["B"], c["N"]

    def rnd(*shape, std=1.0, dtype=None):
        t = torch.randn(shape, generator=g, device="cuda", dtype=dtype or _T[c["dtype"]])
        return t if std == 1.0 else t.mul_(std)

    s["parents"] = _parents(c, g)
    if c["op"] == "verify":
        V = c["V"]
        logits = rnd(B, N, V, std=3.0, dtype=torch.float32)
        s["p"] = torch.softmax(logits, -1).to(_T[c["dtype"]])
        q = torch.softmax(logits.add_(rnd(B, N, V, std=0.7, dtype=torch.float32)), -1)
        del logits
        s["draft"] = q.to(_T[c["dtype"]]) if c["draft"] else None
        up = s["parents"].clamp(min=0).long()
        rows = q.gather(1, up[:, :, None].expand(B, N, V)).view(B * N, V)
        s["tokens"] = torch.multinomial(rows, 1, generator=g).view(B, N).to(torch.int32)
        s["u"] = torch.rand((B, N), generator=g, device="cuda")
        return s
    H, d = c["H"], c["H"] * c["d_k"]
    s["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda") if c["lo"] else None
    K = rnd(B, _stride(c), d)
    s["K"] = _banded(K, H) if c["banded"] else K
    if c["op"] == "commit":
        # a path down the tree that takes about a quarter of the nodes
        keep = torch.rand((B, N), generator=g, device="cuda") < 0.25
        keep[:, 0] = True
        at = torch.arange(N, device="cuda").expand(B, N)
        s["path"] = torch.where(keep, at, torch.full_like(at, N)).sort(-1).values.to(torch.int32)
        s["path"][s["path"] == N] = -1
        s["n_path"] = keep.sum(-1).to(torch.int32)
        return s
    s["W"] = rnd(d, d, std=d ** -0.5)
    s["q"] = rnd(B, N, d, std=1.5)
    if c["rope"]:                                        # cos and sin of every position that a row or node can have
        theta = 10000.0 ** (-2.0 * torch.arange(c["d_k"] // 2, device="cuda", dtype=torch.float64) / c["d_k"])
        ang = torch.arange(c["T"] + N, device="cuda", dtype=torch.float64)[:, None] * theta
        s["rope"] = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()
    else:
        s["rope"] = None
    return s


# ---- plain forms --------------------------------------------------------------------------------------

def _ancestors(par, N):
    """[B][N][N]: whether node j is node i or one of its ancestors; unused slots have no row and no column.  By doubling: six rounds reach 64 nodes."""
    B = par.shape[0]
    i = torch.arange(N, device=par.device)
    par = par.long()
    ok = (par >= -1) & (par < i)
    up = torch.where(ok & (par >= 0), par, i)            # a root points to itself
    eye = torch.eye(N, dtype=torch.bool, device=par.device).expand(B, N, N)
    anc, bad = eye, ~ok
    for _ in range(6):
        anc = anc | anc.gather(1, up[:, :, None].expand(B, N, N))
        bad = bad | bad.gather(1, up)
        up = up.gather(1, up)
    return anc & ~bad[:, :, None] & ~bad[:, None, :], ~bad


def _tree_plain(s, F):
    c = s["c"]
    B, N, H, d_k, T = c["B"], c["N"], c["H"], c["d_k"], c["T"]
    d, R = H * d_k, T + N
    K = _unbanded(s["K"], H) if c["banded"] else s["K"]
    K = K[:, :R].to(F)
    lens = s["lens"].long() if s["lens"] is not None else torch.full((B,), T, device="cuda")
    anc, used = _ancestors(s["parents"], N)
    t = torch.arange(R, device="cuda")
    j = t[None, :] - lens[:, None]                       # node of a row, where 0 <= j < N
    drafted = (j >= 0) & (j < N)
    jc = j.clamp(0, N - 1)
    sees = (j[:, None, :] < 0) | (drafted[:, None, :] & anc.gather(2, jc[:, None, :].expand(B, N, R)))
    sees = sees & used[:, :, None]
    k = K.view(B, R, H, d_k)
    if s["rope"] is not None:
        depth = anc.sum(-1) - 1
        pos = torch.where(drafted, lens[:, None] + depth.gather(1, jc).clamp(min=0), t[None, :]).clamp(max=R - 1)
        cs = s["rope"].to(F)[pos]                        # [B][R][d_k / 2][2]
        co, si = cs[:, :, None, :, 0], cs[:, :, None, :, 1]
        x1, x2 = k[..., 0::2], k[..., 1::2]
        k = torch.stack([x1 * co + x2 * si, x2 * co - x1 * si], -1).reshape(B, R, H, d_k)
    kt = k.permute(0, 2, 3, 1).reshape(B * H, d_k, R)
    q = s["q"].to(F).view(B, N, H, d_k).permute(0, 2, 1, 3).reshape(B * H, N, d_k)
    S = torch.bmm(q, kt).view(B, H, N, R) * (1.0 / math.sqrt(d_k))
    S = S.masked_fill(~sees[:, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    e = torch.exp(S - torch.where(m == -math.inf, torch.zeros_like(m), m))
    del S
    e = e / e.sum(-1, keepdim=True).clamp(min=torch.finfo(F).tiny)
    C = torch.bmm(e.view(B, H * N, R), K).view(B, H, N, d)
    del e
    W = s["W"].to(F).view(d, H, d_k).transpose(0, 1).contiguous()
    out = torch.bmm(C.transpose(0, 1).reshape(H, B * N, d), W)
    return out.view(H, B, N, d_k).permute(1, 2, 0, 3).reshape(B, N, d).to(_T[c["dtype"]] if F == torch.float32 else F)


def _verify_plain(s):
    """The walk goes through the nodes in the order of their numbers, all sequences at once: a node that hangs on the one reached last is tested."""
    c = s["c"]
    B, N, V = c["B"], c["N"], c["V"]
    b = torch.arange(B, device="cuda")
    tok, par, u = s["tokens"].long(), s["parents"].long(), s["u"].double()
    p, q = s["p"], s["draft"]
    cur = torch.zeros(B, dtype=torch.long, device="cuda")
    a = torch.zeros(B, dtype=torch.float64, device="cuda")
    Fa = torch.ones_like(a)
    out = torch.zeros((B, V), dtype=torch.bool, device="cuda")     # tokens that were chosen and rejected
    path = torch.zeros((B, N), dtype=torch.bool, device="cuda")
    path[:, 0] = True
    for i in range(1, N):
        x = tok[:, i]
        px = p[b, cur, x].double()
        child = par[:, i] == cur
        if q is not None:
            qx = q[b, cur, x].double()
            yes = child & (u[:, i] * Fa * qx < px - a * qx)
            no = child & ~yes
            a = torch.where(yes, torch.zeros_like(a), torch.where(no, a + Fa, a))
            cur = torch.where(yes, torch.full_like(cur, i), cur)
            r = (p[b, cur].double() - a[:, None] * q[b, cur].double()).clamp(min=0)
            Fa = torch.where(a == 0, torch.ones_like(a), r.sum(-1))
        else:
            px = torch.where(out[b, x], torch.zeros_like(px), px)
            yes = child & (u[:, i] * Fa < px)
            no = child & ~yes
            Fa = torch.where(yes, torch.ones_like(a), torch.where(no, Fa - px, Fa))
            cur = torch.where(yes, torch.full_like(cur, i), cur)
            out = out & ~yes[:, None]
            out[b, x] = out[b, x] | no
        path[:, i] = yes
    r = p[b, cur].double()
    r = torch.where(out, torch.zeros_like(r), r) if q is None else (r - a[:, None] * q[b, cur].double()).clamp(min=0)
    run_ = r.cumsum(-1)
    over = run_ > u[:, :1] * run_[:, -1:]
    at = torch.arange(V, device="cuda")
    nxt = torch.where(over, at, V).amin(-1)
    last = torch.where(r > 0, at, -1).amax(-1)
    top = p[b, cur].float()
    top = torch.where(top == top.amax(-1, keepdim=True), at, V).amin(-1)
    nxt = torch.where(run_[:, -1] > 0, torch.where(nxt < V, nxt, last), top)
    i = torch.arange(N, device="cuda").expand(B, N)
    n = path.sum(-1)
    order = torch.where(path, i, torch.full_like(i, N)).sort(-1).values
    order = torch.where(order == N, torch.full_like(order, -1), order)
    return {"path": order.to(torch.int32), "n_path": n.to(torch.int32), "next": nxt.to(torch.int32)}


def _commit_plain(s):
    c = s["c"]
    B, N, T, H = c["B"], c["N"], c["T"], c["H"]
    lens = s["lens"].long() if s["lens"] is not None else torch.full((B,), T, device="cuda")
    K = s["K"]
    b = torch.arange(B, device="cuda")[:, None]
    j = torch.arange(N, device="cuda")[None]
    path = s["path"].long()
    there = j < s["n_path"][:, None]
    src, dst = lens[:, None] + torch.where(there, path, j), lens[:, None] + j
    if c["banded"]:
        Kv = K.view(B, -1, H, 32, c["d_k"])
        Kv[b, dst // 32, :, dst % 32] = Kv[b, src // 32, :, src % 32]
    else:
        K[b, dst] = K[b, src]
    return {"K": K, "lens": (lens + s["n_path"]).to(torch.int32)}


def _own(s):
    from paper_2503_05840_amd import binding
    c = s["c"]
    B, N = c["B"], c["N"]
    if c["op"] == "verify":
        path, n_path, nxt = (torch.empty(shape, dtype=torch.int32, device="cuda") for shape in ((B, N), (B,), (B,)))
        binding.slim_tree_verify(s["tokens"], s["parents"], s["p"], s["draft"], s["u"], path, n_path, nxt, B, N, c["V"], dtype=c["dtype"])
        return {"path": path, "n_path": n_path, "next": nxt}
    H, T, d = c["H"], c["T"], c["H"] * c["d_k"]
    kw = dict(dtype=c["dtype"], t_stride=_stride(c), k_layout=binding.K_BANDED if c["banded"] else binding.K_ROWMAJOR)
    if c["op"] == "commit":
        lens = torch.empty((B,), dtype=torch.int32, device="cuda")
        binding.slim_tree_commit(s["K"], s["path"], s["n_path"], lens, B, N, H, T, d, seq_lens=s["lens"], **kw)
        return {"K": s["K"], "lens": lens}
    out = torch.empty((B, N, d), dtype=_T[c["dtype"]], device="cuda")
    binding.slim_tree_decode(s["q"], s["K"], s["W"], s["parents"], out, B, N, H, T, d, seq_lens=s["lens"], rope_table=s["rope"], **kw)
    return out


def run(state):
    if own:
        return _own(state)
    op = state["c"]["op"]
    return _tree_plain(state, torch.float32) if op == "tree" else _verify_plain(state) if op == "verify" else _commit_plain(state)


# ---- the definition in 64 bits ------------------------------------------------------------------------

def exact(case, seed):
    """Row by row from the definition: node by node for the tree's attention (through the values V = K W_KV that the method never stores), on the
    host for verification; a commit computes nothing, its rows are copied one after the other."""
    s = prepare(case, seed)
    c = case
    B, N = c["B"], c["N"]
    par = s["parents"].cpu().tolist()
    if c["op"] == "verify":
        tok, u = s["tokens"].cpu().tolist(), s["u"].double().cpu().tolist()
        paths, count, nxt = [], [], []
        for b in range(B):
            cur, path = 0, [0]
            res = s["p"][b, 0].double().cpu()
            first = True
            while True:
                went = False
                for i in range(cur + 1, N):
                    if par[b][i] != cur:
                        continue
                    x = tok[b][i]
                    if s["draft"] is not None:
                        q = s["draft"][b, cur].double().cpu()
                        total = 1.0 if first else float(res.sum())
                        if u[b][i] * float(q[x]) * total < float(res[x]):
                            went = True
                        else:
                            res = (res - total * q).clamp(min=0)
                    else:
                        total = 1.0 if first else left
                        if u[b][i] * total < float(res[x]):
                            went = True
                        else:
                            left = total - float(res[x])
                            res[x] = 0.0
                    first = False
                    if went:
                        cur = i
                        path.append(i)
                        res = s["p"][b, i].double().cpu()
                        first = True
                        break
                if not went:
                    break
            run_ = res.cumsum(0)
            total = float(run_[-1])
            if total > 0:
                over = torch.nonzero(run_ > u[b][0] * total)
                v = int(over[0]) if len(over) else int(torch.nonzero(res > 0)[-1])
            else:
                v = int(torch.nonzero(s["p"][b, cur] == s["p"][b, cur].max())[0])
            paths.append(path + [-1] * (N - len(path)))
            count.append(len(path))
            nxt.append(v)
        t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        return {"path": t(paths), "n_path": t(count), "next": t(nxt)}
    H, d_k, T = c["H"], c["d_k"], c["T"]
    lens = _lens(c)
    if c["op"] == "commit":
        K = _unbanded(s["K"], H) if c["banded"] else s["K"].clone()
        for b, (path, n) in enumerate(zip(s["path"].cpu().tolist(), s["n_path"].cpu().tolist())):
            for j in range(n):
                if path[j] != j:
                    K[b, lens[b] + j] = K[b, lens[b] + path[j]]
        new = torch.tensor(lens, dtype=torch.int32, device="cuda") + s["n_path"]
        return {"K": _banded(K, H) if c["banded"] else K, "lens": new}
    d = H * d_k
    out = torch.zeros((B, N, d), dtype=torch.float64, device="cuda")
    W = s["W"].double()
    Kall = _unbanded(s["K"], H) if c["banded"] else s["K"]
    for b in range(B):
        L = lens[b]
        rows = Kall[b, :L + N].double()
        # row by row of the sequence: its position, and for every node the rows that it sees
        chains = []
        for i in range(N):
            chain, at = [], i
            while True:
                up = par[b][at]
                if up < -1 or up >= at:
                    chain = None
                    break
                chain.append(at)
                if up < 0:
                    break
                at = up
            chains.append(chain)
        see = torch.zeros((N, L + N), dtype=torch.bool)
        pos = list(range(L)) + [L] * N
        for i, chain in enumerate(chains):
            if chain is not None:
                see[i, :L] = True
                see[i, [L + x for x in chain]] = True
                pos[L + i] = L + len(chain) - 1
        alive = [i for i in range(N) if chains[i] is not None]
        if not alive:
            continue
        see = see[alive].cuda()
        key = rows.clone()
        if s["rope"] is not None:
            table = s["rope"].double()[torch.tensor(pos, device="cuda")]
            pair = rows.view(L + N, H, d_k // 2, 2)
            z = torch.complex(pair[..., 0], pair[..., 1]) * torch.complex(table[..., 0], -table[..., 1])[:, None]
            key = torch.view_as_real(z).reshape(L + N, d)
        for h in range(H):
            cols = slice(h * d_k, (h + 1) * d_k)
            score = s["q"][b, alive, cols].double() @ key[:, cols].t().contiguous() / math.sqrt(d_k)
            w = torch.softmax(score.masked_fill(~see, -math.inf), -1)
            if N <= d_k // 2:
                out[b, alive, cols] = (w @ rows) @ W[:, cols].contiguous()
            else:
                out[b, alive, cols] = w @ (rows @ W[:, cols].contiguous())
    return out
