"""Operators beside the block-sparse path, over the range they are called in: Q and K made ready for attention
(norm and rotation by position), and attention over packed sequences of different lengths, with or without a
long prefix that every sequence shares.

A case is a dict of plain values.  ``kind`` is one of

* ``rotate``: Q ``[B, S, H, 128]`` and K ``[B, S, Hk, 128]`` are normalised (``norm``: per head, over the whole
  token, or not) and rotated by each token's position on ``axes`` axes (``pairs0 .. 2`` rotation pairs each; adjacent
  or half-split pairs); the last ``text`` tokens of a request stand at position 0 of every axis but the first.
* ``attend``: ``N`` sequences in one call, sequence i with n_i queries (``q_lo .. q_hi``) and its keys: ``c_lo ..
  c_hi`` earlier tokens followed by its own n_i (``cross``: the ``c`` tokens alone).  ``H`` query heads share ``Hk``
  key heads.  ``causal``: the last query sees the last key, the one before it one key less.  ``cache``: keys stand
  in a buffer of ``c_hi + q_hi`` rows per sequence instead of end to end.
* ``prefix``: the same, and every query also sees the ``P`` tokens of one shared prefix.

Lengths are spread over their logarithm and follow from the case (``lens``); values follow from the seed alone.
``fresh``: the work plan of the batch is made in the pass (a step's first layer), otherwise it is at hand (its
other layers).
"""

from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
EPS = 1e-6
THETA = 10000.0
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _rotate(B, grid, H, Hk, dtype, norm, pairs, adjacent, text=0, **name):
    T, Y, X = grid
    return dict(name, kind="rotate", B=B, T=T, Y=Y, X=X, text=text, H=H, Hk=Hk, dtype=dtype, norm=norm, axes=len(pairs),
                pairs0=pairs[0], pairs1=pairs[1] if len(pairs) > 1 else 0, pairs2=pairs[2] if len(pairs) > 2 else 0,
                adjacent=adjacent)


def _attend(N, q, c, H, Hk, dtype, causal, P=0, cross=False, cache=False, lse=False, fresh=False, lens=1, **name):
    return dict(name, kind="prefix" if P else "attend", N=N, q_lo=q[0], q_hi=q[1], c_lo=c[0], c_hi=c[1], H=H, Hk=Hk,
                dtype=dtype, causal=causal, P=P, cross=cross, cache=cache, lse=lse, fresh=fresh, lens=lens)


def listed():
    return [
        # the next token of four requests (latency)
        _rotate(4, (1, 1, 1), 32, 8, "f16", "head", (64,), False, name="rotate_next_token_f16"),
        # a 480p 14B layer: norm over the whole token, adjacent pairs on time, height and width
        _rotate(1, (21, 30, 52), 40, 40, "bf16", "token", (22, 21, 21), True, name="rotate_480p_bf16"),
        # a 720p 5B layer with a norm of its own for each head, half-split pairs
        _rotate(1, (31, 22, 40), 24, 24, "bf16", "head", (16, 24, 24), False, name="rotate_720p_bf16"),
        # three small clips with text behind the video tokens, grouped heads, rotation alone, odd sizes
        _rotate(3, (5, 13, 19), 12, 3, "f16", "none", (22, 21, 21), True, text=77, name="rotate_clips_text_f16"),
        # the next token of four requests with short caches (latency)
        _attend(4, (1, 1), (50, 300), 32, 8, "f16", True, cache=True, name="next_token_f16"),
        # a batch of prompts of very different lengths
        _attend(24, (16, 4096), (0, 0), 32, 8, "bf16", True, lse=True, fresh=True, name="prompts_bf16"),
        # one long causal sequence
        _attend(1, (20280, 20280), (0, 0), 40, 8, "bf16", True, name="prompt_long_bf16"),
        # clips of different lengths, every token sees its whole clip
        _attend(5, (1560, 10920), (0, 0), 12, 12, "f16", False, name="clips_f16"),
        # video tokens that attend to their request's text
        _attend(4, (1560, 16380), (20, 512), 24, 24, "bf16", False, cross=True, fresh=True, name="text_cross_bf16"),
        # one step of 64 requests with long caches of different lengths
        _attend(64, (1, 1), (512, 16384), 40, 8, "bf16", True, cache=True, name="next_tokens_long_bf16"),
        # one step of 96 requests behind one prefix
        _attend(96, (1, 1), (1, 512), 32, 8, "bf16", True, P=16384, cache=True, fresh=True, name="prefix_next_tokens_bf16"),
        # eight prompts behind one prefix
        _attend(8, (30, 700), (0, 0), 16, 4, "f16", True, P=6001, lse=True, name="prefix_prompts_f16"),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "prompts", "prompts", "clips", "cross", "step", "step", "prefix", "prefix"])
    dtype = rng.choice(["bf16", "f16"])
    Hk = rng.choice([1, 2, 3, 4, 8, 12])
    H = Hk * rng.choice([1, 1, 2, 4, 5, 8])
    lens, lse, fresh = rng.randint(1, 1 << 20), rng.random() < 0.3, rng.random() < 0.5
    if kind == "rotate":
        S = _log(rng, 1, 40000)
        T = rng.randint(1, min(S, 24))
        Y = max(1, round(math.sqrt(S / T) * rng.uniform(0.6, 0.95)))
        X = max(1, round(S / (T * Y)))
        pairs = rng.choice([(64,), (32, 32), (22, 21, 21), (16, 24, 24), (8, 28, 28)])
        c = _rotate(rng.choice([1, 1, 2, 3, 5]), (T, Y, X), H, Hk, dtype, rng.choice(["none", "head", "token"]), pairs,
                    rng.random() < 0.5, text=rng.choice([0, 0, 77, 200]))
        while work(c)["bytes"] > 1.3e9:
            if c["B"] > 1:
                c["B"] -= 1
            else:
                c["X"] = c["X"] * 3 // 4
        return c
    P = 0
    if kind == "prompts":
        lo = _log(rng, 1, 500)
        q, k = (lo, lo * rng.randint(1, 20)), rng.choice([(0, 0), (0, 0), (1, _log(rng, 2, 4000))])
        c = dict(N=_log(rng, 1, 32), q=q, c=k, causal=True, cache=rng.random() < 0.3)
    elif kind == "clips":
        lo = _log(rng, 200, 6000)
        c = dict(N=rng.randint(1, 6), q=(lo, lo * rng.randint(1, 3)), c=(0, 0), causal=False)
    elif kind == "cross":
        lo = _log(rng, 100, 9000)
        c = dict(N=rng.randint(1, 8), q=(lo, lo * 2), c=(_log(rng, 1, 40), _log(rng, 40, 700)), causal=False, cross=True)
    elif kind == "step":
        c = dict(N=_log(rng, 1, 128), q=(1, rng.choice([1, 1, 1, 4])), c=(_log(rng, 1, 1000), _log(rng, 1000, 30000)),
                 causal=True, cache=rng.random() < 0.7)
    else:
        P = _log(rng, 100, 30000)
        hi = rng.choice([1, 1, 3, 40, 600])
        c = dict(N=_log(rng, 2, 128) if hi < 100 else rng.randint(2, 8), q=(1, hi), c=(0, _log(rng, 2, 800)), causal=True,
                 cache=rng.random() < 0.5)
    c = _attend(H=H, Hk=Hk, dtype=dtype, P=P, lse=lse, fresh=fresh, lens=lens, **c)
    while c["N"] * (c["c_hi"] + c["q_hi"]) * Hk * D > 4e8 or _padded(c) > 1.5e10 or work(c)["flops"] > 4e12:
        if c["N"] > 1:
            c["N"] = c["N"] * 2 // 3
        else:
            c["q_hi"] = max(1, c["q_hi"] * 2 // 3)
            c["q_lo"] = min(c["q_lo"], c["q_hi"])
    return c


def _lengths(case):
    """(queries, keys) of each sequence."""
    rng = random.Random(case["lens"])

    def one(lo, hi):
        return hi if lo >= hi else min(hi, _log(rng, lo + 1, hi + 1) - 1)

    nq = [one(case["q_lo"], case["q_hi"]) for _ in range(case["N"])]
    ctx = [one(case["c_lo"], case["c_hi"]) for _ in range(case["N"])]
    return nq, ctx if case["cross"] else [c + n for c, n in zip(ctx, nq)]


def _padded(case):
    """Scores that the plain form holds."""
    nq, nk = _lengths(case)
    return case["N"] * max(nq) * (max(nk) + case["P"]) * case["H"]


def _pairs(case):
    return [case["pairs%d" % a] for a in range(case["axes"])]


def work(case):
    """Each input read once, each output written once; attention: two products per visible (query, key) pair."""
    if case["kind"] == "rotate":
        tokens = case["B"] * (case["T"] * case["Y"] * case["X"] + case["text"])
        el = tokens * (case["H"] + case["Hk"]) * D
        return {"bytes": 4 * el + 4 * case["axes"] * tokens, "flops": 7 * el}
    nq, nk = _lengths(case)
    seen = 0
    for n, m in zip(nq, nk):
        skip = n - min(n, m)    # queries ahead of the first key
        seen += (n - skip) * m - (n - skip) * (n - skip - 1) // 2 if case["causal"] else n * m
    seen += sum(nq) * case["P"]
    tq, tk = sum(nq), sum(nk) + case["P"]
    return {"bytes": 4 * tq * case["H"] * D + 4 * tk * case["Hk"] * D + 4 * tq * case["H"] * case["lse"],
            "flops": 4 * seen * case["H"] * D}


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------

def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _positions(case):
    """int32 [axes, S]: (t, y, x) of the video tokens, then text tokens that count on along the first axis; with
    fewer axes the token's index (one) or frame and index within it (two)."""
    T, Y, X, text = case["T"], case["Y"], case["X"], case["text"]
    i = torch.arange(T * Y * X, device="cuda")
    cols = {1: [i], 2: [i // (Y * X), i % (Y * X)], 3: [i // (Y * X), i // X % Y, i % X]}[case["axes"]]
    behind = [torch.arange(text, device="cuda") + int(cols[0][-1]) + 1] + [i.new_zeros(text)] * (case["axes"] - 1)
    return torch.stack([torch.cat(p) for p in zip(cols, behind)]).to(torch.int32)


def _freqs(case):
    """Radians per position of the 64 rotation pairs, axis by axis, each with a ladder of its own."""
    return [THETA ** (-i / n) for n in _pairs(case) for i in range(n)]


def _offsets(n):
    return [0] + list(np.cumsum(n))


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def randn(*shape, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dt)

    H, Hk = case["H"], case["Hk"]
    state = {"case": case}
    if case["kind"] == "rotate":
        S = case["T"] * case["Y"] * case["X"] + case["text"]
        state["q"], state["k"] = randn(case["B"], S, H, D, scale=1.7), randn(case["B"], S, Hk, D, scale=0.6)
        state["positions"], state["freqs"] = _positions(case), _freqs(case)
        state["weights"] = None
        if case["norm"] != "none":
            state["weights"] = [1 + 0.2 * torch.randn(*((D,) if case["norm"] == "head" else (h, D)), device="cuda", generator=g)
                                for h in (H, Hk)]
        if own:
            from paper_2606_25040_amd import ops
            state["rotary"] = ops.RotaryAxes(_pairs(case), state["freqs"], adjacent=case["adjacent"])
        return state
    nq, nk = _lengths(case)
    state["nq"], state["nk"] = nq, nk
    state["q"] = randn(sum(nq), H, D, scale=1.5)
    rows = case["c_hi"] + case["q_hi"]
    starts = [rows * i for i in range(case["N"] + 1)] if case["cache"] else _offsets(nk)
    state["k"], state["v"] = randn(starts[-1], Hk, D), randn(starts[-1], Hk, D)
    state["q_offsets"], state["k_offsets"], state["k_lens"] = _ints(_offsets(nq)), _ints(starts), _ints(nk)
    state["prefix"] = (randn(case["P"], Hk, D), randn(case["P"], Hk, D)) if case["P"] else None
    if own:
        state["plan"] = None if case["fresh"] else _plan(state)
    return state


# --------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------

def _plan(state):
    from paper_2606_25040_amd import ops
    case = state["case"]
    return ops.plan_packed_attn(state["q_offsets"], state["k_offsets"], state["q"].shape[0], state["k"].shape[0], case["H"],
                                case["Hk"], causal=case["causal"], k_lens=state["k_lens"] if case["cache"] else None,
                                prefix=case["P"], max_q=max(state["nq"]))


def _own(state):
    from paper_2606_25040_amd import ops
    case = state["case"]
    if case["kind"] == "rotate":
        wq, wk = state["weights"] or (None, None)
        return ops.qk_norm_rope(state["q"], state["k"], rotary=state["rotary"], positions=state["positions"],
                                norm=None if case["norm"] == "none" else case["norm"], q_weight=wq, k_weight=wk, eps=EPS)
    plan = _plan(state) if case["fresh"] else state["plan"]
    pk, pv = state["prefix"] or (None, None)
    return ops.packed_attn_fwd(state["q"], state["k"], state["v"], plan, prefix_k=pk, prefix_v=pv, return_lse=case["lse"])


def _turned(x, weight, norm, cos, sin, adjacent):
    """Norm and rotation of x [B, S, heads, 128] in 32 bits; cos and sin [S, 1, 64]."""
    y = x.float()
    if weight is not None:
        over = (3,) if norm == "head" else (2, 3)
        y = y * torch.rsqrt((y * y).mean(over, keepdim=True) + EPS) * weight
    if adjacent:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(3)
    else:
        a, b = y[..., :D // 2], y[..., D // 2:]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return y.to(x.dtype)


def _rotation(state):
    case = state["case"]
    pairs = _pairs(case)
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"), torch.tensor(pairs, device="cuda"), output_size=D // 2)
    angle = state["positions"].double().t()[:, axis] * torch.tensor(state["freqs"], dtype=torch.float64, device="cuda")
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    weights = state["weights"] or (None, None)
    return [_turned(x, w, case["norm"], cos, sin, case["adjacent"]) for x, w in zip((state["q"], state["k"]), weights)]


def _attention(state):
    """Sequences padded to the longest, a few key heads at a time, in 32 bits."""
    case, nq, nk = state["case"], max(state["nq"]), max(max(state["nk"]), 1)
    N, H, Hk, P = case["N"], case["H"], case["Hk"], case["P"]
    G = H // Hk
    q, k, v = state["q"], state["k"], state["v"]
    q_len, k_len = state["q_offsets"].diff(), state["k_lens"]
    iq, ik = torch.arange(nq, device="cuda"), torch.arange(nk, device="cuda")
    is_q = iq < q_len[:, None]                                                        # [N, nq]
    at_q = (state["q_offsets"][:-1, None] + iq).clamp(max=q.shape[0] - 1)
    at_k = (state["k_offsets"][:-1, None] + torch.minimum(ik, (k_len - 1).clamp(min=0)[:, None])).clamp(max=max(0, k.shape[0] - 1))
    seen = ik < k_len[:, None, None]                                                  # [N, nq, nk]
    if case["causal"]:
        seen = seen & (ik <= (iq + (k_len - q_len)[:, None])[:, :, None])
    seen = seen[:, None, None]
    out, lse = torch.empty_like(q), torch.empty(H, q.shape[0], device="cuda")
    some = max(1, min(Hk, int(2.5e9) // (N * G * nq * (nk + P))))
    for h in range(0, Hk, some):
        e = min(Hk, h + some)
        qh = q[at_q, h * G:e * G].float().reshape(N, nq, e - h, G, D).permute(0, 2, 3, 1, 4) / math.sqrt(D)   # [N, heads, G, nq, D]
        qf = qh.reshape(N, e - h, G * nq, D)
        kh = k[at_k, h:e].float().permute(0, 2, 3, 1).contiguous()                    # [N, heads, D, nk]
        vh = v[at_k, h:e].float().permute(0, 2, 1, 3).contiguous()
        z = torch.matmul(qf, kh).reshape(N, e - h, G, nq, nk)
        z = z.masked_fill_(~seen, -math.inf)
        m = z.amax(-1, keepdim=True)
        if P:
            pk = state["prefix"][0][:, h:e].float().permute(1, 2, 0).contiguous()     # [heads, D, P]
            pv = state["prefix"][1][:, h:e].float().permute(1, 0, 2).contiguous()
            y = torch.matmul(qf, pk).reshape(N, e - h, G, nq, P)
            m = torch.maximum(m, y.amax(-1, keepdim=True))
        safe = torch.where(m == -math.inf, 0.0, m)
        z = z.sub_(safe).exp_()
        l = z.sum(-1, keepdim=True)
        o = torch.matmul(z.reshape(N, e - h, G * nq, nk), vh).reshape(N, e - h, G, nq, D)
        if P:
            y = y.sub_(safe).exp_()
            l = l + y.sum(-1, keepdim=True)
            o = o + torch.matmul(y.reshape(N, e - h, G * nq, P), pv).reshape(N, e - h, G, nq, D)
        o = torch.where(l > 0, o / l, 0.0)
        where = at_q[is_q]
        out[where, h * G:e * G] = o.permute(0, 3, 1, 2, 4).reshape(N, nq, (e - h) * G, D)[is_q].to(out.dtype)
        if case["lse"]:
            s = (safe + l.log()).squeeze(-1).permute(1, 2, 0, 3).reshape((e - h) * G, N, nq)
            lse[h * G:e * G, where] = s[:, is_q]
    return (out, lse) if case["lse"] else out


def run(state):
    if own:
        return _own(state)
    return _rotation(state) if state["case"]["kind"] == "rotate" else _attention(state)


# --------------------------------------------------------------------------------------------------
# the same in 64 bits
# --------------------------------------------------------------------------------------------------

def _exact_rotation(state):
    case = state["case"]
    outs = []
    for n, x in enumerate((state["q"], state["k"])):
        y = x.double()
        B, S, heads, _ = y.shape
        if case["norm"] == "head":
            y = y / (y.pow(2).sum(3, keepdim=True) / D + EPS).sqrt() * state["weights"][n].double()
        elif case["norm"] == "token":
            y = y / (y.pow(2).sum((2, 3), keepdim=True) / (heads * D) + EPS).sqrt() * state["weights"][n].double()
        first = 0
        z = torch.empty_like(y)
        for a, count in enumerate(_pairs(case)):
            for i in range(count):
                p = first + i
                angle = state["positions"][a].double() * state["freqs"][p]
                turn = torch.polar(torch.ones_like(angle), angle)[None, :, None]
                one, two = (2 * p, 2 * p + 1) if case["adjacent"] else (p, p + D // 2)
                w = torch.complex(y[..., one], y[..., two]) * turn
                z[..., one], z[..., two] = w.real, w.imag
            first += count
        outs.append(z)
    return outs


def _exact_attention(state):
    case, q = state["case"], state["q"]
    H, Hk = case["H"], case["Hk"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full((H, q.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    starts = state["k_offsets"].tolist()
    q0 = 0
    for i, (n, m) in enumerate(zip(state["nq"], state["nk"])):
        for j in range(Hk):
            kk, vv = (x[starts[i]:starts[i] + m, j].double() for x in (state["k"], state["v"]))
            if case["P"]:
                kk, vv = (torch.cat((p[:, j].double(), x)) for p, x in zip(state["prefix"], (kk, vv)))
            if kk.shape[0] == 0:
                continue
            kk = kk.t().contiguous()
            step = max(1, int(2e8) // kk.shape[1])
            for h in range(j * (H // Hk), (j + 1) * (H // Hk)):
                for t in range(0, n, step):
                    e = min(n, t + step)
                    z = q[q0 + t:q0 + e, h].double() @ kk / math.sqrt(D)
                    if case["causal"]:
                        last = torch.arange(t, e, device="cuda") + m - n + case["P"]
                        z.masked_fill_(torch.arange(kk.shape[1], device="cuda") > last[:, None], -math.inf)
                    s = torch.logsumexp(z, 1)
                    some = s > -math.inf
                    z.sub_(torch.where(some, s, 0.0)[:, None]).exp_()
                    out[q0 + t:q0 + e, h] = z @ vv
                    lse[h, q0 + t:q0 + e] = s
        q0 += n
    return (out, lse) if case["lse"] else out


def exact(case, seed):
    state = prepare(case, seed)
    return _exact_rotation(state) if case["kind"] == "rotate" else _exact_attention(state)
