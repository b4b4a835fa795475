"""The attention operators' workloads: what a stage's attention sublayer does
between the codec's decompress and the reparameterized output projection.

A case is one pass of one operator of ``paper_2607_13332_amd.ssn``:

* ``norm``: the norms of queries and keys for each head with the position
  rotation in the same pass (``qk_norm_rope``), forward or backward;
* ``append``: the serving form of the same: queries normed and rotated, keys
  normed and rotated on their way into a paged cache, values appended to it
  (``kv_append``);
* ``attn``: attention of the new tokens of a batch of sequences, each a chunk
  at its sequence's end, over the paged cache (``paged_attention``).

``own`` False computes the same from the formulas with elementary torch
operations in 32 bits.  Buffers that a stage keeps from one step to the next
(outputs, caches, page tables, workspaces, the rotation table) are made in
``prepare``.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
THETA = 5e5            # Pluralis-8B's rotation base


def _norm(name, dtype, direction, N, Hq, Hk, D, S, style="halves"):
    return {"name": name, "op": "norm", "dtype": dtype, "dir": direction, "N": N, "Hq": Hq, "Hk": Hk,
            "D": D, "S": S, "style": style}


def _batch(name, op, dtype, kind, B, q, low, high, Hq, Hk, D, page, style="halves"):
    return {"name": name, "op": op, "dtype": dtype, "kind": kind, "B": B, "q": q, "low": low,
            "high": high, "Hq": Hq, "Hk": Hk, "D": D, "page": page, "style": style}


def listed():
    return [
        # Pluralis-8B (40 query heads, 8 key heads of 128), one training
        # sequence of 4096 tokens forward.
        _norm("norm_fwd_paper8b_b1", "bf16", "fwd", 4096, 40, 8, 128, 4096),
        # Three coalesced sequences less their padding tokens, backward.
        _norm("norm_bwd_paper8b_b3_ragged", "bf16", "bwd", 12205, 40, 8, 128, 4096),
        # A small float32 model (as many key heads as query heads, heads of
        # 64, neighbouring pairs rotated), backward.
        _norm("norm_bwd_f32", "f32", "bwd", 2011, 16, 16, 64, 1024, style="pairs"),
        # One sequence's next token: the smallest call, latency counts.
        _batch("append_token_b1", "append", "bf16", "token", 1, 1, 2011, 2011, 40, 8, 128, 64),
        # A batch of single tokens with caches of all lengths, float32.
        _batch("append_token_b64_f32", "append", "f32", "token", 64, 1, 1, 4096, 32, 8, 128, 64),
        # Prompts of several sequences, ragged, small pages.
        _batch("append_prompts_b4", "append", "bf16", "prompt", 4, 4096, 900, 4096, 40, 8, 128, 16),
        # One sequence's next token over a middling cache.
        _batch("attn_token_b1", "attn", "bf16", "token", 1, 1, 2011, 2011, 40, 8, 128, 64),
        # A serving batch: 64 next tokens, caches of all lengths.
        _batch("attn_token_b64", "attn", "bf16", "token", 64, 1, 1, 4096, 40, 8, 128, 64),
        # Few sequences with long caches.
        _batch("attn_token_long", "attn", "bf16", "token", 4, 1, 100_001, 131_072, 32, 8, 128, 64),
        # A whole prompt of the model's sequence length.
        _batch("attn_prompt_4096", "attn", "bf16", "prompt", 1, 4096, 4096, 4096, 40, 8, 128, 64),
        # A chunk of a prompt and many next tokens in one batch, small pages.
        _batch("attn_mixed_b32", "attn", "bf16", "mixed", 32, 517, 300, 8192, 32, 8, 128, 16),
        # Prompts in float32, heads of 64, a key head for each query head.
        _batch("attn_prompts_f32", "attn", "f32", "prompt", 3, 1024, 300, 1024, 16, 16, 64, 16),
    ]


# Most work of one drawn case: that of the largest listed ones.
MOST_BYTES = 1.9e9
MOST_FLOPS = 1.7e11
MOST_FLOPS_F32 = 1e10


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    while True:
        dtype = rng.choices(("bf16", "f32"), (3, 1))[0]
        Hq, Hk, D = rng.choice(((40, 8, 128), (32, 8, 128), (32, 4, 128), (16, 16, 64), (32, 8, 64),
                                (20, 4, 128), (14, 2, 64)))
        style = rng.choice(("halves", "pairs"))
        op = rng.choices(("norm", "append", "attn"), (3, 2, 5))[0]
        if op == "norm":
            case = _norm(None, dtype, rng.choice(("fwd", "bwd")), _log(rng, 500, 12288), Hq, Hk, D,
                         rng.choice((1024, 2048, 4096)), style)
        else:
            kind = rng.choices(("token", "prompt", "chunk", "mixed"), (3, 2, 2, 2))[0]
            B = _log(rng, 1, 64) if kind in ("token", "mixed") else _log(rng, 1, 8)
            high = _log(rng, 100, 131072 if kind == "token" else 32768 if kind == "chunk" else 8192)
            low = rng.randint(1, high)
            q = 1 if kind == "token" else high if kind == "prompt" else _log(rng, 1, min(1024, high))
            case = _batch(None, op, dtype, kind, B, q, low, high, Hq, Hk, D,
                          rng.choice((16, 16, 64, 64, 128, rng.randint(8, 96))), style)
        del case["name"]
        w = work(case)
        cache = 0 if op == "norm" else 2 * sum(_lengths(case)[1]) * Hk * D * _size(dtype)
        if max(w["bytes"], cache) <= MOST_BYTES and \
                w["flops"] <= (MOST_FLOPS_F32 if dtype == "f32" else MOST_FLOPS):
            return case


# --------------------------------------------------------------------------
# Inputs: lengths from the case, values from the seed.
# --------------------------------------------------------------------------
def _dt(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _size(dtype):
    return 4 if dtype == "f32" else 2


def _lengths(case):
    """New tokens and length (those included) of each sequence of a batch:
    the first one has the most of both."""
    B, q, low, high, kind = case["B"], case["q"], case["low"], case["high"], case["kind"]
    rng = random.Random(f"{kind} {B} {q} {low} {high}")
    new, lens = [], []
    for b in range(B):
        length = high if b == 0 else rng.randint(low, high)
        if kind == "token":
            n = 1
        elif kind == "prompt":
            n = length
        elif kind == "chunk":
            n = min(length, q if b == 0 else rng.randint(1, q))
        else:                         # one chunk among single tokens
            n = q if b == 0 else 1
        new.append(n)
        lens.append(length)
    return new, lens


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 29)
    return g


def _normal(g, shape, dtype, std=1.0):
    """N(0, std^2) values in `dtype`, drawn in slabs of rows."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    rows = max(1, 2 ** 26 // max(1, math.prod(shape[1:])))
    for r in range(0, shape[0], rows):
        part = out[r:r + rows]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV) * std)
    return out


def _table(P, R):
    """Row p: cos(p f_i), then sin(p f_i), f_i = THETA^(-2 i / R), i < R / 2."""
    f = torch.pow(torch.tensor(THETA, dtype=torch.float64, device=DEV),
                  torch.arange(0, R, 2, dtype=torch.float64, device=DEV) / -R)
    a = torch.arange(P, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _heads(rows, first, heads, D):
    """Heads [first, first + heads) of packed rows, as [N, heads, D] (a view
    of what the layer's one projection for queries, keys and values gives)."""
    return rows[:, first * D:(first + heads) * D].view(rows.shape[0], heads, D)


def _weight(g, D, t):
    return (1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(t)


def _inputs(case, seed):
    g, t = _gen(seed), _dt(case["dtype"])
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    s = {}
    if case["op"] == "norm":
        N, S = case["N"], case["S"]
        s["rows"] = _normal(g, (N, (Hq + 2 * Hk) * D), t)
        s["wq"], s["wk"] = _weight(g, D, t), _weight(g, D, t)
        s["table"] = _table(S, D)
        s["pos"] = (torch.arange(N, device=DEV) % S).to(torch.int32)
        if case["dir"] == "bwd":
            s["GQ"], s["GK"] = _normal(g, (N, Hq, D), t), _normal(g, (N, Hk, D), t)
        return s
    new, lens = _lengths(case)
    N, S, B = sum(new), case["page"], case["B"]
    width = -(-max(lens) // S)
    need = [-(-n // S) for n in lens]
    # pages were handed out in no order; what the table holds past a
    # sequence's last page is not used
    order = torch.randperm(sum(need), generator=g, device=DEV).to(torch.int32)
    s["pages"] = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        s["pages"][b, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["Kc"] = _normal(g, (sum(need), Hk, S, D), t)
    s["Vc"] = _normal(g, (sum(need), Hk, S, D), t)
    if case["op"] == "append":
        s["rows"] = _normal(g, (N, (Hq + 2 * Hk) * D), t)
        s["wq"], s["wk"] = _weight(g, D, t), _weight(g, D, t)
        s["table"] = _table(max(lens), D)
    else:
        # normed and rotated queries and keys: scores of a trained model
        # reach further than those of independent normal values
        s["Q"] = _normal(g, (N, Hq, D), t, 1.5)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    t, Hq, Hk, D = _dt(case["dtype"]), case["Hq"], case["Hk"], case["D"]
    if "rows" in s:
        s["Q"] = _heads(s["rows"], 0, Hq, D)
        s["K"] = _heads(s["rows"], Hq, Hk, D)
        s["V"] = _heads(s["rows"], Hq + Hk, Hk, D)
    N = s["Q"].shape[0]
    if case["op"] == "norm" and case["dir"] == "bwd":
        # the gradient of the packed rows; attention's backward writes the values' part
        s["grows"] = torch.zeros((N, (Hq + 2 * Hk) * D), dtype=t, device=DEV)
        s["GQin"], s["GKin"] = _heads(s["grows"], 0, Hq, D), _heads(s["grows"], Hq, Hk, D)
        s["Gwq"] = torch.empty(D, dtype=torch.float32, device=DEV)
        s["Gwk"] = torch.empty(D, dtype=torch.float32, device=DEV)
    else:
        s["Qout"] = torch.empty((N, Hq, D), dtype=t, device=DEV)
    if case["op"] == "norm":
        s["Kout"] = torch.empty((N, Hk, D), dtype=t, device=DEV)
    else:
        s["new"], s["lengths"] = _lengths(case)
    s["ws"] = None
    if own:
        from paper_2607_13332_amd import ssn
        if case["op"] == "norm" and case["dir"] == "bwd":
            s["ws"] = ssn.qk_norm_rope_workspace(N, Hq, Hk, D, DEV, dtype=t)
        if case["op"] == "attn":
            s["ws"] = ssn.paged_attention_workspace(N, case["B"], Hq, Hk, D, max(s["new"]),
                                                    max(s["lengths"]), DEV, dtype=t)
    return s


# --------------------------------------------------------------------------
# The plain forms, in 32 bits.
# --------------------------------------------------------------------------
def _rotate(x, cs, style, sign=1.0):
    """x [N, H, D] turned by the angles whose cosines and sines are cs [N, D]
    (sign -1: turned back)."""
    h = x.shape[-1] // 2
    c, s = cs[:, None, :h], cs[:, None, h:] * sign
    if style == "halves":
        a, b = x[..., :h], x[..., h:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)


def _norm_rope(x, w, cs, style):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return _rotate(x * r * w.float(), cs, style)


def _norm_rope_backward(x, w, cs, style, gy):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    g = _rotate(gy.float(), cs, style, -1.0)
    h = g * w.float()
    return r * (h - n * (h * n).mean(-1, keepdim=True)), (g * n).sum((0, 1))


def _positions(s):
    """Sequence and position of every new token."""
    starts, lens = s["starts"].long(), s["lens"].long()
    i = torch.arange(s["Q"].shape[0], device=DEV)
    b = torch.searchsorted(starts[1:], i, right=True)
    return b, lens[b] - (starts[b + 1] - i)


def _gather(cache, pages, length):
    """Cache rows 0 .. length of one sequence, [Hk, length, D] in 32 bits."""
    S = cache.shape[2]
    rows = cache[pages[:-(-length // S)].long()]
    return rows.transpose(0, 1).reshape(cache.shape[1], -1, cache.shape[3])[:, :length].float()


def _attend(q, k, v, length):
    """q [n, Hq, D], the last n tokens of a sequence; k, v [Hk, length, D]."""
    n, Hq, D = q.shape
    Hk = k.shape[0]
    kt = k.transpose(1, 2).contiguous()
    out = torch.empty((n, Hq, D), dtype=torch.float32, device=DEV)
    step = max(1, 2 ** 28 // (Hq * length))
    for i in range(0, n, step):
        part = q[i:i + step].float()
        m = part.shape[0]
        rows = part.view(m, Hk, Hq // Hk, D).permute(1, 0, 2, 3).reshape(Hk, -1, D)
        score = torch.matmul(rows, kt).view(Hk, m, Hq // Hk, length) * D ** -0.5
        at = torch.arange(length - n + i, length - n + i + m, device=DEV)
        hidden = torch.arange(length, device=DEV)[None, :] > at[:, None]
        score = score.masked_fill(hidden[None, :, None, :], -math.inf)
        p = torch.exp(score - score.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(Hk, -1, length), v).view(Hk, m, Hq // Hk, D)
        out[i:i + step] = o.permute(1, 0, 2, 3).reshape(m, Hq, D)
    return out


def _run_plain(s):
    case = s["case"]
    t, style = _dt(case["dtype"]), case["style"]
    if case["op"] == "norm":
        cs = s["table"][s["pos"].long()]
        if case["dir"] == "fwd":
            s["Qout"].copy_(_norm_rope(s["Q"], s["wq"], cs, style))
            s["Kout"].copy_(_norm_rope(s["K"], s["wk"], cs, style))
            return {"Q": s["Qout"], "K": s["Kout"]}
        gq, gwq = _norm_rope_backward(s["Q"], s["wq"], cs, style, s["GQ"])
        gk, gwk = _norm_rope_backward(s["K"], s["wk"], cs, style, s["GK"])
        s["GQin"].copy_(gq)
        s["GKin"].copy_(gk)
        return {"GQ": s["GQin"], "GK": s["GKin"], "Gwq": gwq, "Gwk": gwk}
    if case["op"] == "append":
        b, p = _positions(s)
        cs, S = s["table"][p], case["page"]
        s["Qout"].copy_(_norm_rope(s["Q"], s["wq"], cs, style))
        page = s["pages"].long()[b, p // S]
        s["Kc"][page, :, p % S] = _norm_rope(s["K"], s["wk"], cs, style).to(t)
        s["Vc"][page, :, p % S] = s["V"]
        return {"Q": s["Qout"], "Kc": s["Kc"], "Vc": s["Vc"]}
    at = 0
    for b, (n, length) in enumerate(zip(s["new"], s["lengths"])):
        k, v = _gather(s["Kc"], s["pages"][b], length), _gather(s["Vc"], s["pages"][b], length)
        s["Qout"][at:at + n] = _attend(s["Q"][at:at + n], k, v, length)
        at += n
    return {"O": s["Qout"]}


def run(state):
    s = state
    if not own:
        return _run_plain(s)
    from paper_2607_13332_amd import ssn
    case = s["case"]
    style = case["style"]
    if case["op"] == "norm":
        if case["dir"] == "fwd":
            Q, K = ssn.qk_norm_rope(s["Q"], s["K"], s["pos"], s["table"], wq=s["wq"], wk=s["wk"],
                                    eps=EPS, style=style, Qout=s["Qout"], Kout=s["Kout"])
            return {"Q": Q, "K": K}
        GQ, GK, Gwq, Gwk = ssn.qk_norm_rope_backward(
            s["Q"], s["K"], s["GQ"], s["GK"], s["pos"], s["table"], wq=s["wq"], wk=s["wk"], eps=EPS,
            style=style, GQin=s["GQin"], GKin=s["GKin"], Gwq=s["Gwq"], Gwk=s["Gwk"], workspace=s["ws"])
        return {"GQ": GQ, "GK": GK, "Gwq": Gwq, "Gwk": Gwk}
    if case["op"] == "append":
        Q = ssn.kv_append(s["K"], s["V"], s["Kc"], s["Vc"], s["pages"], s["starts"], s["lens"],
                          Q=s["Q"], table=s["table"], wq=s["wq"], wk=s["wk"], eps=EPS, style=style,
                          Qout=s["Qout"])
        return {"Q": Q, "Kc": s["Kc"], "Vc": s["Vc"]}
    O = ssn.paged_attention(s["Q"], s["Kc"], s["Vc"], s["pages"], s["starts"], s["lens"],
                            max(s["new"]), max(s["lengths"]), out=s["Qout"], workspace=s["ws"])
    return {"O": O}


def work(case):
    Hq, Hk, D, s = case["Hq"], case["Hk"], case["D"], _size(case["dtype"])
    if case["op"] == "norm":
        N = case["N"]
        act = N * (Hq + Hk) * D * s
        table = 4 * min(N, case["S"]) * D + 4 * N
        if case["dir"] == "fwd":
            return {"bytes": 2 * act + table + 2 * D * s, "flops": 9.0 * N * (Hq + Hk) * D}
        return {"bytes": 3 * act + table + 2 * D * (s + 4), "flops": 16.0 * N * (Hq + Hk) * D}
    new, lens = _lengths(case)
    N = sum(new)
    index = 4 * (2 * case["B"] + 1) + 4 * sum(-(-n // case["page"]) for n in lens)
    if case["op"] == "append":
        spots = len({p for n, length in zip(new, lens) for p in range(length - n, length)})
        entries = 4 * sum(-(-length // case["page"]) - (length - n) // case["page"]
                          for n, length in zip(new, lens))
        return {"bytes": 2 * N * (Hq + 2 * Hk) * D * s + 4 * spots * D + entries + 8 * case["B"] + 2 * D * s,
                "flops": 9.0 * N * (Hq + Hk) * D}
    seen = sum(n * (length - n) + n * (n + 1) // 2 for n, length in zip(new, lens))
    return {"bytes": 2 * N * Hq * D * s + 2 * sum(lens) * Hk * D * s + index,
            "flops": 4.0 * seen * Hq * D}


# --------------------------------------------------------------------------
# The definitions in 64 bits.
# --------------------------------------------------------------------------
def _turn(style, cs):
    """The rotation as complex numbers: how rows become them and back."""
    h = cs.shape[-1] // 2
    z = torch.complex(cs[:, :h].double(), cs[:, h:].double())[:, None, :]
    if style == "halves":
        return z, lambda x: torch.complex(x[..., :h], x[..., h:]), lambda y: torch.cat([y.real, y.imag], -1)
    return (z, lambda x: torch.view_as_complex(x.unflatten(-1, (h, 2)).contiguous()),
            lambda y: torch.view_as_real(y).flatten(-2))


def _exact_forward(x, w, cs, style):
    x = x.double()
    z, pack, unpack = _turn(style, cs)
    rms = (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
    return unpack(pack(x / rms * w.double()) * z)


def _exact_backward(x, w, cs, style, gy):
    x, w = x.double(), w.double()
    D = x.shape[-1]
    z, pack, unpack = _turn(style, cs)
    g = unpack(pack(gy.double()) * z.conj())
    rms = (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt()
    dot = (g * w * x).sum(-1, keepdim=True)
    return g * w / rms - x * dot / (D * rms.pow(3)), (g * x / rms).sum((0, 1))


def exact(case, seed):
    s = _inputs(case, seed)
    Hq, Hk, D, style = case["Hq"], case["Hk"], case["D"], case["style"]
    if "rows" in s:
        N = s["rows"].shape[0]
        heads = s["rows"].view(N, Hq + 2 * Hk, D)
        Q, K, V = heads[:, :Hq], heads[:, Hq:Hq + Hk], heads[:, Hq + Hk:]
    if case["op"] == "norm":
        cs = s["table"][s["pos"].long()]
        if case["dir"] == "fwd":
            return {"Q": _exact_forward(Q, s["wq"], cs, style), "K": _exact_forward(K, s["wk"], cs, style)}
        gq, gwq = _exact_backward(Q, s["wq"], cs, style, s["GQ"])
        gk, gwk = _exact_backward(K, s["wk"], cs, style, s["GK"])
        return {"GQ": gq, "GK": gk, "Gwq": gwq, "Gwk": gwk}
    new, lens = _lengths(case)
    S = case["page"]
    if case["op"] == "append":
        pos = torch.cat([torch.arange(length - n, length) for n, length in zip(new, lens)]).to(DEV)
        seq = torch.cat([torch.full((n,), b) for b, n in enumerate(new)]).to(DEV)
        cs = s["table"][pos]
        slot = s["pages"][seq, pos // S].long() * S + pos % S
        caches = []
        for cache, rows in ((s["Kc"], _exact_forward(K, s["wk"], cs, style)), (s["Vc"], V.double())):
            c = cache.double().transpose(1, 2).reshape(-1, Hk, D)      # one row of heads a slot
            c[slot] = rows
            caches.append(c.view(-1, S, Hk, D).transpose(1, 2).contiguous())
        return {"Q": _exact_forward(Q, s["wq"], cs, style), "Kc": caches[0], "Vc": caches[1]}
    G, at = Hq // Hk, 0
    O = torch.empty((sum(new), Hq, D), dtype=torch.float64, device=DEV)
    for b, (n, length) in enumerate(zip(new, lens)):
        t = torch.arange(length, device=DEV)
        page, off = s["pages"][b, t // S].long(), t % S
        for h in range(Hk):
            k, v = s["Kc"][page, h, off].double(), s["Vc"][page, h, off].double()
            kt = k.t().contiguous()
            for j in range(G):
                for i in range(0, n, 1024):
                    q = s["Q"][at + i:at + min(n, i + 1024), h * G + j].double()
                    score = (q @ kt) / math.sqrt(D)
                    last = torch.arange(length - n + i, length - n + i + q.shape[0], device=DEV)
                    score[t[None, :] > last[:, None]] = -math.inf
                    O[at + i:at + i + q.shape[0], h * G + j] = torch.softmax(score, -1) @ v
        at += n
    return {"O": O}
