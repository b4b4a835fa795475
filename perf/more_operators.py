"""The 4-bit cache's workloads: a stage's paged key/value cache held in 4 bits an
element, from the append to the attention that reads it.

A case is one pass of one of these operators of ``paper_2607_13332_amd.ssn``:

* ``append``: keys (normed and rotated, as ``qk_norm_rope`` leaves them) and
  values of a batch's new tokens are quantised into the cache
  (``kv_append_fp4``) and read back (``kv_read_fp4``): what the tokens after
  them will see of them;
* ``read``: whole sequences are read back, as a program does that moves them to
  a cache of another type or shares a prefix (``kv_read_fp4``);
* ``attn``: attention of the new tokens of a batch of sequences, each a chunk
  at its sequence's end, over the 4-bit cache (``paged_attention_fp4``).

32 consecutive elements of a head share a power of two 2^e, e the smallest with
which the largest of them rounds to at most 6, and each is held as the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 with its sign, ties to the even code.  A byte of
codes [pages, Hk, page_size, D / 2] holds two elements, the first in the low
half; a byte of scales [pages, Hk, page_size, D / 32] holds e + 127.

``own`` False computes the same from the formulas with elementary torch
operations in 32 bits.  Buffers that a stage keeps from one step to the next
(outputs, caches, page tables, workspaces) are made in ``prepare``.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
GROUP = 32             # elements that share a scale
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, op, dtype, kind, B, q, low, high, Hq, Hk, D, page):
    return {"name": name, "op": op, "dtype": dtype, "kind": kind, "B": B, "q": q, "low": low, "high": high,
            "Hq": Hq, "Hk": Hk, "D": D, "page": page}


def listed():
    return [
        # One sequence's next token of a model with 8 key heads of 128: the
        # smallest call, latency counts.
        _case("append_token_b1", "append", "bf16", "token", 1, 1, 2011, 2011, 40, 8, 128, 64),
        # A batch of single tokens with caches of all lengths, float32.
        _case("append_token_b64_f32", "append", "f32", "token", 64, 1, 1, 4096, 32, 8, 128, 64),
        # Prompts of several sequences, ragged, small pages.
        _case("append_prompts_b4", "append", "bf16", "prompt", 4, 4096, 900, 4096, 40, 8, 128, 16),
        # Sequences of all lengths that move to a bf16 cache.
        _case("read_b8", "read", "bf16", "prompt", 8, 8192, 1, 8192, 40, 8, 128, 64),
        # A prefix in float32, a key head for each query head, an odd page size.
        _case("read_b1_f32", "read", "f32", "prompt", 1, 1501, 1501, 1501, 16, 16, 64, 24),
        # One sequence's next token over a middling cache.
        _case("attn_token_b1", "attn", "bf16", "token", 1, 1, 2011, 2011, 40, 8, 128, 64),
        # A serving batch: 64 next tokens, caches of all lengths.
        _case("attn_token_b64", "attn", "bf16", "token", 64, 1, 1, 4096, 40, 8, 128, 64),
        # Few sequences with long caches.
        _case("attn_token_long", "attn", "bf16", "token", 4, 1, 100_001, 131_072, 32, 8, 128, 64),
        # A whole prompt of the model's sequence length.
        _case("attn_prompt_4096", "attn", "bf16", "prompt", 1, 4096, 4096, 4096, 40, 8, 128, 64),
        # A chunk of a long prompt, by far the most of it in the cache already.
        _case("attn_chunk_long", "attn", "bf16", "chunk", 1, 512, 32_768, 32_768, 32, 8, 128, 64),
        # A chunk of a prompt and many next tokens in one batch, small pages.
        _case("attn_mixed_b32", "attn", "bf16", "mixed", 32, 517, 300, 8192, 32, 8, 128, 16),
        # Prompts in float32, heads of 64, a key head for each query head.
        _case("attn_prompts_f32", "attn", "f32", "prompt", 3, 1024, 300, 1024, 16, 16, 64, 16),
    ]


# Most work of one drawn case: that of the largest listed ones.
MOST_BYTES = 5.6e8
MOST_FLOPS = 2.8e11
MOST_FLOPS_F32 = 1e10
MOST_SCORES = 3e9      # that a pass computes, the hidden ones of its longest sequences among them


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    while True:
        dtype = rng.choices(("bf16", "f32"), (3, 1))[0]
        Hq, Hk, D = rng.choice(((40, 8, 128), (32, 8, 128), (32, 4, 128), (16, 16, 64), (32, 8, 64),
                                (20, 4, 128), (14, 2, 64), (12, 4, 96), (8, 2, 256)))
        op = rng.choices(("append", "read", "attn"), (3, 2, 6))[0]
        kind = rng.choices(("token", "prompt", "chunk", "mixed"), (3, 2, 2, 2))[0]
        if op == "read":
            kind = "prompt"
        B = _log(rng, 1, 64) if kind in ("token", "mixed") else _log(rng, 1, 8)
        high = _log(rng, 100, 131072 if kind == "token" else 32768 if kind == "chunk" else 8192)
        low = rng.randint(1, high)
        q = 1 if kind == "token" else high if kind == "prompt" else _log(rng, 1, min(1024, high))
        page = rng.choice((16, 16, 64, 64, 128, rng.randint(8, 96)))
        case = _case(None, op, dtype, kind, B, q, low, high, Hq, Hk, D, page)
        del case["name"]
        w = work(case)
        cache = 2 * sum(_lengths(case)[1]) * Hk * _held(D)
        scores = 0 if op != "attn" else Hq * sum(len(g) * n * t for g, n, t in _alike(case))
        if max(w["bytes"], cache) <= MOST_BYTES and scores <= MOST_SCORES and \
                w["flops"] <= (MOST_FLOPS_F32 if dtype == "f32" else MOST_FLOPS):
            return case


# --------------------------------------------------------------------------
# Inputs: lengths from the case, values from the seed.
# --------------------------------------------------------------------------
def _dt(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _size(dtype):
    return 4 if dtype == "f32" else 2


def _held(D):
    """Bytes of a head of D elements in the cache."""
    return D // 2 + D // GROUP


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


def _alike(case):
    """The sequences with a single new token and the others: (sequences, most
    new tokens, greatest length) of each that there is."""
    new, lens = _lengths(case)
    groups = ([b for b, n in enumerate(new) if n == 1], [b for b, n in enumerate(new) if n > 1])
    return [(g, max(new[b] for b in g), max(lens[b] for b in g)) for g in groups if g]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 53)
    return g


def _slabs(rows, width):
    step = max(1, 2 ** 26 // max(1, width))
    return [(r, min(rows, r + step)) for r in range(0, rows, step)]


def _normal(g, shape, dtype, std=1.0):
    """N(0, std^2) values in `dtype`, drawn in slabs of rows."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    for a, b in _slabs(shape[0], math.prod(shape[1:])):
        out[a:b] = torch.randn((b - a, *shape[1:]), generator=g, device=DEV) * std
    return out


def _held_normal(g, shape):
    """Codes and scales of N(0, 1) values."""
    *lead, D = shape
    codes = torch.empty((*lead, D // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((*lead, D // GROUP), dtype=torch.uint8, device=DEV)
    for a, b in _slabs(shape[0], math.prod(shape[1:])):
        codes[a:b], scales[a:b] = _quantise(torch.randn((b - a, *shape[1:]), generator=g, device=DEV))
    return codes, scales


def _inputs(case, seed):
    g, t = _gen(seed), _dt(case["dtype"])
    Hq, Hk, D, S, B = case["Hq"], case["Hk"], case["D"], case["page"], case["B"]
    new, lens = _lengths(case)
    N, s = sum(new), {}
    need = [-(-n // S) for n in lens]
    # pages were handed out in no order; what the table holds past a
    # sequence's last page is not used
    order = torch.randperm(sum(need), generator=g, device=DEV).to(torch.int32)
    s["pages"] = torch.full((B, max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        s["pages"][b, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    shape = (sum(need), Hk, S, D)
    if case["op"] == "append":
        # what the layer's norm and rotation leave of keys, and the part of its
        # one projection that holds the values
        s["K"] = _normal(g, (N, Hk, D), t)
        s["V"] = _normal(g, (N, 2 * Hk * D), t)[:, Hk * D:].view(N, Hk, D)
        for c in "KV":
            s[c + "c"] = torch.zeros((*shape[:3], D // 2), dtype=torch.uint8, device=DEV)
            s[c + "s"] = torch.zeros((*shape[:3], D // GROUP), dtype=torch.uint8, device=DEV)
        return s
    s["Kc"], s["Ks"] = _held_normal(g, shape)
    s["Vc"], s["Vs"] = _held_normal(g, shape)
    if case["op"] == "attn":
        # normed and rotated queries and keys: scores of a trained model
        # reach further than those of independent normal values
        s["Q"] = _normal(g, (N, Hq, D), t, 1.5)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    t, Hq, Hk, D = _dt(case["dtype"]), case["Hq"], case["Hk"], case["D"]
    new, lens = _lengths(case)
    N = sum(new)
    s["most"] = (max(new), max(lens))
    if case["op"] != "attn":
        s["Kout"] = torch.empty((N, Hk, D), dtype=t, device=DEV)
        s["Vout"] = torch.empty((N, Hk, D), dtype=t, device=DEV)
        return s
    s["O"] = torch.empty((N, Hq, D), dtype=t, device=DEV)
    # the sequences of each kind, and where their rows are
    s["groups"] = []
    at = [0]
    for n in new:
        at.append(at[-1] + n)
    for g, n, length in _alike(case):
        rows = torch.cat([torch.arange(at[b], at[b + 1]) for b in g]).to(DEV)
        s["groups"].append((torch.tensor(g, device=DEV), rows, n, length))
    s["ws"] = None
    if own:
        from paper_2607_13332_amd import ssn
        s["ws"] = ssn.paged_attention_fp4_workspace(N, case["B"], Hq, Hk, D, *s["most"], DEV, dtype=t)
    return s


# --------------------------------------------------------------------------
# The plain forms, in 32 bits.
# --------------------------------------------------------------------------
def _quantise(x):
    """Codes [.., D / 2] and scales [.., D / 32] of x [.., D]."""
    x = x.float().unflatten(-1, (-1, GROUP))
    # max = m 2^E with 1/2 <= m < 1: 8 m 2^(E - 3), and from 7 on it rounds to 8
    m, E = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = (E - 3 + (m >= 0.875)).clamp(-126, 125)
    e = torch.where(m == 0, -126, e)
    v = x.abs() * torch.pow(2.0, -e.float())
    code = ((v > 0.25).to(torch.uint8) + (v >= 0.75) + (v > 1.25) + (v >= 1.75) + (v > 2.5) + (v >= 3.5) + (v > 5.0)
            + (x < 0).to(torch.uint8) * 8)
    code = code.flatten(-2)
    return (code[..., 0::2] | (code[..., 1::2] << 4)), (e + 127).squeeze(-1).to(torch.uint8)


def _values(codes, scales):
    """The values that codes and scales stand for, in 32 bits."""
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=DEV)
    pair = torch.stack([level.repeat(16), level.repeat_interleave(16)], 1)       # of a byte
    x = pair[codes.long()].flatten(-2).unflatten(-1, (-1, GROUP))
    return (x * torch.pow(2.0, scales.float() - 127)[..., None]).flatten(-2)


def _rows_at(s):
    """Page and place in it of every row's position."""
    starts, lens = s["starts"].long(), s["lens"].long()
    i = torch.arange(s["Kout"].shape[0], device=DEV)
    b = torch.searchsorted(starts[1:], i, right=True)
    p = lens[b] - (starts[b + 1] - i)
    S = s["case"]["page"]
    return s["pages"].long()[b, p // S], p % S


def _gathered(s, name, seqs, length):
    """Positions 0 .. length - 1 of the sequences, [B, Hk, length, D]; past a
    sequence's end whatever a page holds."""
    S = s["case"]["page"]
    pages = s["pages"][seqs, :-(-length // S)].clamp(min=0).long()
    x = _values(s[name + "c"][pages], s[name + "s"][pages])                      # [B, pages, Hk, S, D]
    return x.transpose(1, 2).flatten(2, 3)[:, :, :length]


def _attend(s, seqs, rows, n, length):
    """The outputs of the sequences' rows (at most n each): all of them as wide
    as the widest."""
    case = s["case"]
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    B, G = seqs.shape[0], Hq // Hk
    starts, lens = s["starts"].long(), s["lens"].long()
    first, last = starts[seqs], starts[seqs + 1]
    i = (first[:, None] + torch.arange(n, device=DEV)).clamp(max=s["Q"].shape[0] - 1)
    q = s["Q"][i].float().view(B, n, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, n * G, D)
    score = torch.matmul(q, _gathered(s, "K", seqs, length).transpose(2, 3)) * D ** -0.5
    at = lens[seqs][:, None] - (last[:, None] - i)
    hidden = torch.arange(length, device=DEV) > at[..., None]                    # [B, n, length]
    score = score.view(B, Hk, n, G, length).masked_fill_(hidden[:, None, :, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = (p / p.sum(-1, keepdim=True)).view(B, Hk, n * G, length)
    o = torch.matmul(p, _gathered(s, "V", seqs, length)).view(B, Hk, n, G, D)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    b = torch.searchsorted(last, rows, right=True)
    return o[b, rows - first[b]]


def _run_plain(s):
    case = s["case"]
    if case["op"] == "attn":
        for seqs, rows, n, length in s["groups"]:
            s["O"][rows] = _attend(s, seqs, rows, n, length).to(s["O"].dtype)
        return {"O": s["O"]}
    page, off = _rows_at(s)
    if case["op"] == "append":
        for c in "KV":
            s[c + "c"][page, :, off], s[c + "s"][page, :, off] = _quantise(s[c])
    for c in "KV":
        s[c + "out"].copy_(_values(s[c + "c"][page, :, off], s[c + "s"][page, :, off]))
    return {"K": s["Kout"], "V": s["Vout"]}


def run(state):
    s = state
    if not own:
        return _run_plain(s)
    from paper_2607_13332_amd import ssn
    case = s["case"]
    cache = (s["Kc"], s["Ks"], s["Vc"], s["Vs"], s["pages"], s["starts"], s["lens"])
    if case["op"] == "attn":
        return {"O": ssn.paged_attention_fp4(s["Q"], *cache, *s["most"], out=s["O"], workspace=s["ws"])}
    if case["op"] == "append":
        ssn.kv_append_fp4(s["K"], s["V"], *cache, eps=None)
    K, V = ssn.kv_read_fp4(*cache, s["Kout"].shape[0], Kout=s["Kout"], Vout=s["Vout"])
    return {"K": K, "V": V}


def work(case):
    Hq, Hk, D, t = case["Hq"], case["Hk"], case["D"], _size(case["dtype"])
    new, lens = _lengths(case)
    N = sum(new)
    entries = 4 * sum(-(-length // case["page"]) - (length - n) // case["page"] for n, length in zip(new, lens))
    index = 4 * (2 * case["B"] + 1) + (4 * sum(-(-n // case["page"]) for n in lens) if case["op"] == "attn" else entries)
    if case["op"] == "append":        # in, to the cache, and out again
        return {"bytes": 2 * N * Hk * (2 * D * t + _held(D)) + index, "flops": 12.0 * N * Hk * D}
    if case["op"] == "read":
        return {"bytes": 2 * N * Hk * (D * t + _held(D)) + index, "flops": 2.0 * N * Hk * D}
    seen = sum(n * (length - n) + n * (n + 1) // 2 for n, length in zip(new, lens))
    return {"bytes": 2 * N * Hq * D * t + 2 * sum(lens) * Hk * _held(D) + index, "flops": 4.0 * seen * Hq * D}


# --------------------------------------------------------------------------
# The definitions in 64 bits.
# --------------------------------------------------------------------------
def _exact_held(x):
    """What the cache holds of x [N, Hk, D]: for each element the nearest of all
    levels of its group, by its distance to every one of them."""
    out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=DEV)
    # as far as an odd code is as far as an even one and a little
    odd = torch.arange(8, device=DEV) % 2 * 2.0 ** -40
    for a, b in _slabs(x.shape[0], 16 * math.prod(x.shape[1:])):
        part = x[a:b].double().unflatten(-1, (-1, GROUP))
        top = part.abs().amax(-1, keepdim=True)
        e = torch.where(top > 0, torch.floor(torch.log2(top / 7)) + 1, -126).clamp(-126, 125)
        unit = torch.exp2(e)
        far = (part.abs() / unit)[..., None].sub(level).abs() + odd
        out[a:b] = (level[far.argmin(-1)] * unit * torch.where(part < 0, -1.0, 1.0)).flatten(-2)
    return out


def _exact_values(codes, scales):
    """codes [.., D / 2], scales [.., D / 32] by their bits: sign, two of the
    exponent (0: no leading one), one of the fraction."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    exponent, fraction = (c >> 1) & 3, (c & 1).double()
    size = torch.where(exponent > 0, torch.ldexp(1 + fraction / 2, exponent - 1), fraction / 2)
    size = torch.where(c > 7, -size, size)
    return torch.ldexp(size, scales.int().repeat_interleave(GROUP, -1) - 127)


def exact(case, seed):
    s = _inputs(case, seed)
    Hq, Hk, D, S = case["Hq"], case["Hk"], case["D"], case["page"]
    if case["op"] == "append":
        return {"K": _exact_held(s["K"]), "V": _exact_held(s["V"])}
    new, lens = _lengths(case)
    if case["op"] == "read":
        out = {}
        for c in "KV":
            parts = []
            for b, length in enumerate(lens):
                t = torch.arange(length, device=DEV)
                page, off = s["pages"][b, t // S].long(), t % S
                parts.append(_exact_values(s[c + "c"][page, :, off], s[c + "s"][page, :, off]))
            out[c] = torch.cat(parts)
        return out
    G, at = Hq // Hk, 0
    O = torch.empty((sum(new), Hq, D), dtype=torch.float64, device=DEV)
    for b, (n, length) in enumerate(zip(new, lens)):
        t = torch.arange(length, device=DEV)
        page, off = s["pages"][b, t // S].long(), t % S
        for h in range(Hk):
            k = _exact_values(s["Kc"][page, h, off], s["Ks"][page, h, off])
            v = _exact_values(s["Vc"][page, h, off], s["Vs"][page, h, off])
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
