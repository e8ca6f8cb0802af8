"""The calls that take a prompt into a K-cache held in 4 or 8 bits and generate from it, and the same in plain torch: attention over whole
prompts, rows quantised as the cache is written, rows read back, and the decode step over such a cache.

A case is a plain dict.  `op` says which operator; the other entries:
  prompt  B sequences packed one after the other, T the longest, lo (0: all have T rows; else they spread from lo to T), chunk (0: queries for all rows;
          else for the last `chunk` rows of each sequence: a prompt taken in pieces), H, H_kv, d_k, dtype, causal, fused (q, k and v lie in
          one buffer, row by row beside each other)
  append  B sequences whose caches have T rows, of which lo..T - n are held; n new rows each (ragged: from 1 to n), d, bits, dtype of the rows; what was written is
          read back, for the values it stands for
  read    B sequences' first rows, T at most (ragged: from lo), d, bits, dtype
  decode  B, H, d_k, T, lo, bits, dtype (queries, weights and result), rope (keys carry rotary positions)

A cache's codes are [B][S][d * bits / 8], S the rows kept a sequence (a multiple of 64), column 2 j of a 4-bit row in the low half of byte j; its scales are
[B][d / 32][S] bytes, 127 + the exponent of the power of two that 32 columns share (255: none of them is a number).

Values are random, on the scale that a trained layer has them: unit keys with a few columns that are larger throughout, weights of variance
1 / fan-in, queries whose scores spread by one or two.
"""
import math

import torch

own = False

_T = {"bf16": torch.bfloat16, "f32": torch.float32}


def _prompt(name, B, T, H, H_kv, d_k, lo=0, chunk=0, dtype="bf16", causal=True, fused=False):
    return {"name": name, "op": "prompt", "B": B, "T": T, "H": H, "H_kv": H_kv, "d_k": d_k, "lo": lo, "chunk": chunk, "dtype": dtype,
            "causal": causal, "fused": fused}


def _append(name, B, T, n, d, bits, lo=0, dtype="bf16", ragged=False):
    return {"name": name, "op": "append", "B": B, "T": T, "n": n, "d": d, "bits": bits, "lo": lo, "dtype": dtype, "ragged": ragged}


def _read(name, B, T, d, bits, lo=0, dtype="bf16"):
    return {"name": name, "op": "read", "B": B, "T": T, "d": d, "bits": bits, "lo": lo, "dtype": dtype}


def _decode(name, B, H, d_k, T, bits, lo=0, dtype="bf16", rope=False):
    return {"name": name, "op": "decode", "B": B, "H": H, "d_k": d_k, "T": T, "bits": bits, "lo": lo, "dtype": dtype, "rope": rope}


def listed():
    return [
        # one chat turn on a 7B-shaped layer, odd length, q, k and v as one product leaves them
        _prompt("prompt chat", 1, 777, 32, 32, 128, fused=True),
        # prompts of a serving batch packed together, grouped heads
        _prompt("prompt packed grouped", 8, 4000, 32, 8, 128, lo=90),
        # the largest: the same layer over its whole context
        _prompt("prompt 16k", 1, 16384, 32, 32, 128),
        # a piece of a long prompt behind its cached prefix
        _prompt("prompt piece", 2, 8000, 24, 24, 96, lo=5000, chunk=300),
        # an encoder in full precision: every row sees every other
        _prompt("prompt encoder f32", 4, 1500, 20, 20, 64, dtype="f32", causal=False),
        # the rows of one generated token for a batch: latency
        _append("append tokens", 16, 2048, 1, 4096, 4, lo=500),
        # the rows of a long packed prompt
        _append("append prompt", 4, 8192, 8000, 4096, 4, lo=0, ragged=True),
        # a prefix back for another piece of its prompt, and a batch's in full precision
        _read("read prefix", 1, 7777, 4096, 8),
        _read("read ragged f32", 16, 1500, 1280, 4, lo=100, dtype="f32"),
        # one token of one sequence: short odd context, and the layer's whole context
        _decode("decode short", 1, 32, 128, 777, 4),
        _decode("decode 16k", 1, 32, 128, 16384, 4),
        # rotary keys in 8 bits, ragged contexts of a chat batch
        _decode("decode rotary ragged", 16, 24, 96, 5000, 8, lo=600, rope=True),
    ]


def _spread(n, lo, hi):
    """n lengths: hi, or from lo to hi in a fixed order that is neither sorted nor periodic."""
    if not lo or lo >= hi:
        return [hi] * n
    return [hi] + [lo + int((hi - lo) * (b * 0.6180339887498949 % 1.0)) for b in range(1, n)]


def _new_rows(c):
    return _spread(c["B"], 1, c["n"]) if c["ragged"] and c["n"] > 1 else [c["n"]] * c["B"]


def _held(c):
    """append: rows that each cache holds before the call."""
    return _spread(c["B"], c["lo"], c["T"] - c["n"]) if c["lo"] else [0] * c["B"]


def _stride(T):
    return (T + 63) // 64 * 64


def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def work(case):
    """prompt: q, k, v and the result once, two products for every pair of a query and a key that it sees.  append: the rows once, codes and scales written and read,
    the values written.  read: codes, scales and values once.  decode: codes, scales, W_KV, q and the result once; scores, sums and projection."""
    c = case
    z = _esize(c)
    if c["op"] == "prompt":
        keys = _spread(c["B"], c["lo"], c["T"])
        queries = [min(c["chunk"], n) if c["chunk"] else n for n in keys]
        pairs = sum(m * n - m * (m - 1) // 2 if c["causal"] else m * n for m, n in zip(queries, keys))
        return {"bytes": 2 * (sum(queries) * c["H"] + sum(keys) * c["H_kv"]) * c["d_k"] * z, "flops": 4 * c["d_k"] * c["H"] * pairs}
    held = c["bits"] / 8 + 1 / 32
    if c["op"] == "append":
        n = sum(_new_rows(c)) * c["d"]
        return {"bytes": int(n * (2 * z + 2 * held)), "flops": 0}
    if c["op"] == "read":
        n = sum(_spread(c["B"], c["lo"], c["T"])) * c["d"]
        return {"bytes": int(n * (z + held)), "flops": 0}
    d, n = c["H"] * c["d_k"], sum(_spread(c["B"], c["lo"], c["T"]))
    return {"bytes": int(n * d * held) + d * d * z + 2 * c["B"] * d * z, "flops": 2 * n * d + 2 * n * c["H"] * d + 2 * c["B"] * d * d}


def _cost(c):
    w = work(c)
    rate = 5e14 if c["dtype"] == "bf16" else 5e13
    return max(w["bytes"] / 4e12, w["flops"] / rate)


def draw(rng):
    """One more call from the same ranges: a listed kind with other sizes, odd ones among them."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["prompt", "prompt", "prompt", "prompt f32", "append", "read", "decode", "decode", "decode f32"])
        bits = rng.choice([4, 4, 8])
        if kind.startswith("prompt"):
            f32 = kind == "prompt f32"
            H, H_kv, d_k = rng.choice([(8, 8, 64), (16, 16, 64), (20, 20, 64), (12, 4, 80), (10, 2, 36)] if f32 else
                                      [(32, 32, 128), (32, 32, 128), (32, 8, 128), (28, 4, 128), (40, 40, 128), (16, 2, 128), (24, 24, 96), (20, 20, 64),
                                       (32, 4, 64), (32, 32, 80), (12, 12, 72), (16, 16, 112), (32, 32, 32)])
            T = spread(1, 3000 if f32 else 14000)
            c = _prompt("", spread(1, 4 if f32 else 16), T, H, H_kv, d_k, lo=rng.choice([0, max(1, T // 30)]), chunk=rng.choice([0, 0, 0, spread(1, 600)]),
                        dtype="f32" if f32 else "bf16", causal=rng.random() < 0.8, fused=rng.random() < 0.4)
            if sum(_spread(c["B"], c["lo"], T)) * (H + 2 * H_kv) * d_k > 1 << 28 or H * T * (c["chunk"] or T) > 1 << 33:
                continue
        elif kind == "append":
            n = spread(1, 6000)
            T = n + spread(60, 4000)
            c = _append("", spread(1, 32), T, n, rng.choice([4096, 1280, 2304, 640, 5120, 864]), bits, lo=rng.choice([0, max(1, (T - n) // 5)]),
                        dtype=rng.choice(["bf16", "bf16", "f32"]), ragged=rng.random() < 0.6)
            if c["B"] * T * c["d"] > 1 << 28:
                continue
        elif kind == "read":
            T = spread(1, 12000)
            c = _read("", spread(1, 32), T, rng.choice([4096, 1280, 2304, 640, 5120, 864]), bits, lo=rng.choice([0, max(1, T // 8)]),
                      dtype=rng.choice(["bf16", "bf16", "f32"]))
            if c["B"] * T * c["d"] > 1 << 28:
                continue
        else:
            f32 = kind == "decode f32"
            H, d_k = rng.choice([(8, 64), (12, 80), (16, 64)]) if f32 else rng.choice([(32, 128), (24, 96), (20, 64), (32, 80), (16, 128), (40, 128), (12, 72), (32, 64)])
            T = spread(1, 3000 if f32 else 20000)
            c = _decode("", spread(1, 8 if f32 else 40), H, d_k, T, bits, lo=rng.choice([0, max(1, T // 6)]), dtype="f32" if f32 else "bf16", rope=rng.random() < 0.35)
            if c["B"] * T * H * d_k > 3 << 28 or (f32 and c["B"] * T * H * H * d_k > 1 << 32):
                continue
        if _cost(c) <= most:
            return {k: v for k, v in c.items() if k != "name"}


# ---- the format ---------------------------------------------------------------------------------------

_TOP = {4: (2, 1, 0, 6.0), 8: (8, 3, -6, 448.0)}      # largest exponent, bits of the significand, smallest exponent, largest value


def _pow2(e, F):
    """2^e for whole e from -300 to 300, in two factors (one alone leaves the range of 32 bits)."""
    h = torch.div(e, 2, rounding_mode="floor")
    one = torch.ones((), dtype=F, device=e.device)
    return torch.ldexp(one, h), torch.ldexp(one, e - h)


def _quantised(x, bits):
    """x [..., d] in 32 bits -> (codes one a byte, exponent + 127) of groups of 32 columns."""
    emax, m, emin, top = _TOP[bits]
    g = x.float().unflatten(-1, (-1, 32))
    amax = g.abs().amax(-1)
    sound = torch.isfinite(g).all(-1)
    f, e = torch.frexp(torch.where(sound, amax, torch.ones_like(amax)))         # amax = f 2^e, 0.5 <= f < 1
    s = (e - 1 + (f > 0.875).int() - emax).clamp(min=-127, max=127 - emax)
    s = torch.where(amax == 0, torch.full_like(s, -127), s)
    a, b = _pow2(-s, torch.float32)
    y = g.abs() * a[..., None] * b[..., None]
    _, ye = torch.frexp(y)
    ye = torch.where(y == 0, torch.full_like(ye, emin), ye - 1).clamp(min=emin, max=emax)
    n = torch.round(torch.ldexp(y, m - ye))                                      # in steps of its binade, ties to even
    n = torch.where(torch.ldexp(n, ye - m) > top, torch.full_like(n, round(math.ldexp(top, m - emax))), n).to(torch.int32)
    code = n + (ye - emin) * (1 << m)                                            # (a full binade of steps runs over into the next one's codes)
    code = code + torch.signbit(g).int() * (8 if bits == 4 else 128)
    code = torch.where(sound[..., None], code, torch.zeros_like(code))
    s = torch.where(sound, s + 127, torch.full_like(s, 255))
    return code.flatten(-2), s


def _values(code, s, bits, F):
    """The other way: codes [..., d] one a byte, s [..., d / 32] -> values in F."""
    emax, m, emin, _ = _TOP[bits]
    code, s = code.int(), s.int()
    mag = code & (7 if bits == 4 else 127)
    e = (mag >> m).clamp(min=1)
    n = torch.where(mag >> m > 0, (mag & ((1 << m) - 1)) + (1 << m), mag)
    v = torch.ldexp(n.to(F), e - 1 + emin - m)
    v = torch.where(code >= (8 if bits == 4 else 128), -v, v).unflatten(-1, (-1, 32))
    if bits == 8:
        v = torch.where(mag.unflatten(-1, (-1, 32)) == 127, torch.full_like(v, math.nan), v)
    a, b = _pow2(s - 127, F)
    v = v * a[..., None] * b[..., None]
    return torch.where((s == 255)[..., None], torch.full_like(v, math.nan), v).flatten(-2)


def _packed(code, bits):
    code = code.to(torch.uint8)
    return code if bits == 8 else code[..., 0::2] | (code[..., 1::2] << 4)


def _unpacked(codes, bits):
    return codes if bits == 8 else torch.stack([codes & 15, codes >> 4], -1).flatten(-2)


# ---- inputs -------------------------------------------------------------------------------------------

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"c": c}
    t = _T[c["dtype"]]
    B = c["B"]

    def rnd(*shape, std=1.0):
        x = torch.randn(shape, generator=g, device="cuda", dtype=t)
        return x if std == 1.0 else x.mul_(std)

    def keys(*shape):
        """Unit rows; a few columns are larger throughout."""
        d = shape[-1]
        big = 1.0 + 5.0 * (torch.rand(d, generator=g, device="cuda") < 0.02)
        return rnd(*shape).mul_(big.to(t))

    if c["op"] == "prompt":
        n_k = _spread(B, c["lo"], c["T"])
        n_q = [min(c["chunk"], n) if c["chunk"] else n for n in n_k]
        s["n_q"], s["n_k"] = n_q, n_k
        s["cu_q"] = _ints(_offsets(n_q))
        s["cu_k"] = _ints(_offsets(n_k)) if c["chunk"] else None
        e, e_kv = c["H"] * c["d_k"], c["H_kv"] * c["d_k"]
        if c["fused"] and not c["chunk"]:
            x = rnd(sum(n_q), e + 2 * e_kv)
            x[:, :e].mul_(1.5)
            s["q"], s["k"], s["v"] = x[:, :e], x[:, e:e + e_kv], x[:, e + e_kv:]
        else:
            s["q"], s["k"], s["v"] = rnd(sum(n_q), e, std=1.5), rnd(sum(n_k), e_kv), rnd(sum(n_k), e_kv)
        return s
    d = c["d"] if "d" in c else c["H"] * c["d_k"]
    bits, S = c["bits"], _stride(c["T"])
    if c["op"] == "append":
        new = _new_rows(c)
        s["new"], s["held_list"] = new, _held(c)
        s["rows"] = keys(sum(new), d)
        s["cu"] = _ints(_offsets(new)) if c["ragged"] else None
        s["held"] = _ints(s["held_list"]) if c["lo"] else None
        s["codes"] = torch.zeros((B, S, d * bits // 8), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.zeros((B, d // 32, S), dtype=torch.uint8, device="cuda")
        return s
    # a cache that holds T rows of every sequence; those behind a sequence's length are of no account
    s["codes"] = torch.empty((B, S, d * bits // 8), dtype=torch.uint8, device="cuda")
    s["scales"] = torch.empty((B, d // 32, S), dtype=torch.uint8, device="cuda")
    for b in range(B):
        for at in range(0, S, 8192):
            code, sc = _quantised(keys(min(8192, S - at), d), bits)
            s["codes"][b, at:at + 8192] = _packed(code, bits)
            s["scales"][b, :, at:at + 8192] = sc.t().to(torch.uint8)
    lens = _spread(B, c["lo"], c["T"])
    s["lens_list"] = lens
    if c["op"] == "read":
        s["cu"] = _ints(_offsets(lens)) if c["lo"] else None
        return s
    s["lens"] = _ints(lens) if c["lo"] else None
    s["W"] = rnd(d, d, std=d ** -0.5)
    s["q"] = rnd(B, d, std=1.2)
    s["rope"] = None
    if c["rope"]:                                        # cos and sin of every position
        theta = 10000.0 ** (-2.0 * torch.arange(c["d_k"] // 2, device="cuda", dtype=torch.float64) / c["d_k"])
        ang = torch.arange(c["T"], device="cuda", dtype=torch.float64)[:, None] * theta
        s["rope"] = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()
    return s


# ---- plain forms --------------------------------------------------------------------------------------

def _softmax(S):
    m = S.amax(-1, keepdim=True)
    e = torch.exp(S - torch.where(m == -math.inf, torch.zeros_like(m), m))
    return e / e.sum(-1, keepdim=True).clamp(min=torch.finfo(S.dtype).tiny)


def _prompt_plain(s):
    c = s["c"]
    H, H_kv, d_k = c["H"], c["H_kv"], c["d_k"]
    q = s["q"].float().unflatten(-1, (H_kv, H // H_kv, d_k))
    k, v = s["k"].float().unflatten(-1, (H_kv, d_k)), s["v"].float().unflatten(-1, (H_kv, d_k))
    out = torch.empty((q.shape[0], H_kv, H // H_kv, d_k), dtype=_T[c["dtype"]], device="cuda")
    at_q = at_k = 0
    for m, n in zip(s["n_q"], s["n_k"]):
        if c["causal"]:
            hidden = torch.arange(n, device="cuda") > torch.arange(m, device="cuda")[:, None] + (n - m)
        for h in range(H_kv):                            # one key head after the other: their scores together do not fit
            kt = k[at_k:at_k + n, h].t().contiguous()
            for r in range(H // H_kv):
                S = (q[at_q:at_q + m, h, r] @ kt).mul_(1.0 / math.sqrt(d_k))
                if c["causal"]:
                    S.masked_fill_(hidden, -math.inf)
                out[at_q:at_q + m, h, r] = (_softmax(S) @ v[at_k:at_k + n, h]).to(out.dtype)
        at_q, at_k = at_q + m, at_k + n
    return out.flatten(1)


def _append_plain(s):
    c = s["c"]
    bits = c["bits"]
    out = torch.empty_like(s["rows"])
    at = 0
    for b, (n, held) in enumerate(zip(s["new"], s["held_list"])):
        code, sc = _quantised(s["rows"][at:at + n], bits)
        s["codes"][b, held:held + n] = _packed(code, bits)
        s["scales"][b, :, held:held + n] = sc.t().to(torch.uint8)
        out[at:at + n] = _values(code, sc, bits, torch.float32).to(out.dtype)
        at += n
    return out


def _rows_plain(s, b, n):
    bits = s["c"]["bits"]
    return _values(_unpacked(s["codes"][b, :n], bits), s["scales"][b, :, :n].t(), bits, torch.float32)


def _read_plain(s):
    return torch.cat([_rows_plain(s, b, n).to(_T[s["c"]["dtype"]]) for b, n in enumerate(s["lens_list"])])


def _decode_plain(s):
    c = s["c"]
    H, d_k = c["H"], c["d_k"]
    d = H * d_k
    out = torch.empty((c["B"], d), dtype=_T[c["dtype"]], device="cuda")
    W = s["W"].float().view(d, H, d_k).transpose(0, 1).contiguous()
    for b, n in enumerate(s["lens_list"]):
        K = _rows_plain(s, b, n)
        k = K.view(n, H, d_k)
        if s["rope"] is not None:
            co, si = s["rope"][:n, None, :, 0], s["rope"][:n, None, :, 1]
            x1, x2 = k[..., 0::2], k[..., 1::2]
            k = torch.stack([x1 * co + x2 * si, x2 * co - x1 * si], -1).flatten(-2)
        q = s["q"][b].float().view(1, H, d_k)
        p = _softmax((k * q).sum(-1).t() * (1.0 / math.sqrt(d_k)))
        out[b] = torch.bmm((p @ K)[:, None], W).view(d).to(out.dtype)
    return out


def _own(s):
    from paper_2503_05840_amd import binding
    c = s["c"]
    B, T, t = c["B"], c["T"], _T[c["dtype"]]
    if c["op"] == "prompt":
        out = torch.empty((s["q"].shape[0], c["H"] * c["d_k"]), dtype=t, device="cuda")
        return binding.slim_prompt_attention(s["q"], s["k"], s["v"], s["cu_q"], out, B, c["H"], c["H_kv"], c["d_k"], cu_k=s["cu_k"],
                                             causal=c["causal"], dtype=c["dtype"])
    if c["op"] == "append":
        binding.slim_quant_append(s["rows"], s["codes"], s["scales"], B, T, c["d"], c["bits"], cu_rows=s["cu"], dtype=c["dtype"], seq_lens=s["held"],
                                  t_stride=_stride(T))
        out = torch.empty_like(s["rows"])
        return binding.slim_quant_read(s["codes"], s["scales"], out, B, T, c["d"], c["bits"], cu_rows=s["cu"], dtype=c["dtype"], seq_lens=s["held"],
                                       t_stride=_stride(T))
    if c["op"] == "read":
        out = torch.empty((sum(s["lens_list"]), c["d"]), dtype=t, device="cuda")
        return binding.slim_quant_read(s["codes"], s["scales"], out, B, T, c["d"], c["bits"], cu_rows=s["cu"], dtype=c["dtype"], t_stride=_stride(T))
    d = c["H"] * c["d_k"]
    out = torch.empty((B, d), dtype=t, device="cuda")
    return binding.slim_quant_decode(s["q"], s["codes"], s["scales"], s["W"], out, B, c["H"], T, d, c["bits"], dtype=c["dtype"], seq_lens=s["lens"],
                                     t_stride=_stride(T), rope_table=s["rope"])


def run(state):
    if own:
        return _own(state)
    return {"prompt": _prompt_plain, "append": _append_plain, "read": _read_plain, "decode": _decode_plain}[state["c"]["op"]](state)


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _nearest(x, bits):
    """Rows as the format holds them, from its list of values: the next value below and above, the nearer one, the one of even code between two."""
    if bits == 4:
        grid = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    else:
        grid = [m / 512 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1]
    grid = torch.tensor(grid, dtype=torch.float64, device=x.device)
    g = x.double().reshape(x.shape[0], -1, 32)
    amax = g.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(amax.clamp(min=1e-300)))
    e = torch.where(2.0 ** e > amax, e - 1, torch.where(2.0 ** (e + 1) <= amax, e + 1, e))
    e = torch.where(amax > 1.75 * 2.0 ** e, e + 1, e)
    top = 2 if bits == 4 else 8
    unit = 2.0 ** (e - top).clamp(min=-127, max=127 - top)
    y = (g.abs() / unit).clamp(max=float(grid[-1]))
    hi = torch.searchsorted(grid, y.contiguous()).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    below, above = y - grid[lo], grid[hi] - y
    pick = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return (grid[pick] * unit * torch.sign(g)).reshape(x.shape)


def _from_bytes(s, b, n):
    """The first n rows of a cache from a table of the values of all codes."""
    bits = s["c"]["bits"]
    if bits == 4:
        half = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
        table = half + [-v for v in half]
        by = s["codes"][b, :n].long()
        code = torch.empty((n, 2 * by.shape[1]), dtype=torch.long, device=by.device)
        code[:, 0::2], code[:, 1::2] = by % 16, by // 16
    else:
        half = [(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)]
        table = half[:127] + [math.nan] + [-v for v in half[:127]] + [math.nan]
        code = s["codes"][b, :n].long()
    sc = s["scales"][b, :, :n].t().double()
    unit = torch.where(sc == 255, math.nan, 2.0 ** (sc - 127))
    v = torch.tensor(table, dtype=torch.float64, device=code.device)[code]
    return (v.view(n, -1, 32) * unit[:, :, None]).view(n, -1)


def exact(case, seed):
    """From the definitions: softmax row block by row block for prompts, the list of values for the format, complex numbers for rotations."""
    s = prepare(case, seed)
    c = case
    if c["op"] == "append":
        out = torch.empty(s["rows"].shape, dtype=torch.float64, device="cuda")
        for at in range(0, len(out), 4096):
            out[at:at + 4096] = _nearest(s["rows"][at:at + 4096], c["bits"])
        return out
    if c["op"] == "read":
        return torch.cat([_from_bytes(s, b, n) for b, n in enumerate(s["lens_list"])])
    H, d_k = c["H"], c["d_k"]
    d = H * d_k
    if c["op"] == "prompt":
        out = torch.zeros((sum(s["n_q"]), d), dtype=torch.float64, device="cuda")
        q0 = k0 = 0
        for m, n in zip(s["n_q"], s["n_k"]):
            for h in range(H):
                kv = slice(h * c["H_kv"] // H * d_k, (h * c["H_kv"] // H + 1) * d_k)
                k, v = s["k"][k0:k0 + n, kv].double(), s["v"][k0:k0 + n, kv].double()
                for i in range(0, m, 4096):
                    j = min(i + 4096, m)
                    seen = n - m + j if c["causal"] else n       # (more than the block's first rows see: masked)
                    S = s["q"][q0 + i:q0 + j, h * d_k:(h + 1) * d_k].double() @ k[:seen].t().contiguous() / math.sqrt(d_k)
                    if c["causal"]:
                        row = torch.arange(i, j, device="cuda")[:, None]
                        S = S.masked_fill(torch.arange(seen, device="cuda") - row > n - m, -math.inf)
                    out[q0 + i:q0 + j, h * d_k:(h + 1) * d_k] = torch.softmax(S, -1) @ v[:seen]
            q0, k0 = q0 + m, k0 + n
        return out
    out = torch.zeros((c["B"], d), dtype=torch.float64, device="cuda")
    W = s["W"].double()
    for b, n in enumerate(s["lens_list"]):
        K = _from_bytes(s, b, n)
        key = K
        if c["rope"]:
            table = s["rope"][:n].double()
            z = torch.view_as_complex(K.view(n, H, d_k // 2, 2)) * torch.complex(table[..., 0], -table[..., 1])[:, None]
            key = torch.view_as_real(z).reshape(n, d)
        for h in range(H):
            cols = slice(h * d_k, (h + 1) * d_k)
            w = torch.softmax(key[:, cols] @ s["q"][b, cols].double() / math.sqrt(d_k), 0)
            out[b, cols] = (w @ K) @ W[:, cols]
    return out
