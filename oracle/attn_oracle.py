"""Float64 oracle of the attention sublayer (numpy on the host; definitions
only): norms of heads with the position rotation and their gradients, appends
to a paged cache, attention over it.  Stored inputs (float32, or bfloat16 bit
patterns in uint16) widen exactly."""
from __future__ import annotations

import numpy as np

from oracle.ssn_oracle import f64 as widen


def rope_angles(P: int, R: int, theta: float) -> np.ndarray:
    """[P, R/2] angles p theta^(-2i/R)."""
    return np.arange(P, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(R // 2) / max(R, 1))


def rope_table(P: int, R: int, theta: float) -> np.ndarray:
    a = rope_angles(P, R, theta)
    return np.concatenate([np.cos(a), np.sin(a)], axis=1)


def _rotate(x, rows, style, back=False):
    """x [N, H, D]; rows [N, R] table rows (cosines, then sines)."""
    R = rows.shape[1]
    y = x.copy()
    c = rows[:, None, :R // 2]
    s = rows[:, None, R // 2:] * (-1.0 if back else 1.0)
    first, second = (slice(0, R // 2), slice(R // 2, R)) if style == "halves" else \
        (slice(0, R, 2), slice(1, R, 2))
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    return y


def _prep(x, w, pos, table, D):
    x = widen(x)
    w = np.ones(D) if w is None else widen(w)
    rows = np.zeros((x.shape[0], 0)) if table is None else widen(table)[np.asarray(pos)]
    return x, w, rows


def norm_rope(x, w=None, pos=None, table=None, eps=1e-6, style="halves") -> np.ndarray:
    """x [N, H, D] -> rot(norm(x)); eps None: no norm; table None: no rotation."""
    x, w, rows = _prep(x, w, pos, table, x.shape[-1])
    if eps is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return _rotate(x, rows, style)


def norm_rope_backward(x, gy, w=None, pos=None, table=None, eps=1e-6, style="halves"):
    """(dL/dx, dL/dw) for gy = dL/dy."""
    x, w, rows = _prep(x, w, pos, table, x.shape[-1])
    g = _rotate(widen(gy), rows, style, back=True)
    if eps is None:
        return g, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n, h = x * r, g * w
    return r * (h - n * (h * n).mean(-1, keepdims=True)), (g * n).sum((0, 1))


def batch_rows(starts, lens):
    """(row, sequence, position) of every new token of a batch."""
    for b in range(len(lens)):
        for i in range(starts[b], starts[b + 1]):
            yield i, b, int(lens[b]) - (int(starts[b + 1]) - i)


def gather(cache, pages, length):
    """Cache rows of positions 0 .. length of one sequence, [Hk, length, D]."""
    S = cache.shape[2]
    t = np.arange(length)
    return widen(cache[np.asarray(pages)[t // S], :, t % S]).transpose(1, 0, 2)


def paged_attention(Q, Kc, Vc, pages, starts, lens, scale):
    """(O [N, Hq, D], lse [N, Hq], M [N, Hq, D]) with M the same sum over
    |V|; rows outside every sequence stay NaN."""
    Q = widen(Q)
    N, Hq, D = Q.shape
    Hk = Kc.shape[1]
    O, M = np.full((N, Hq, D), np.nan), np.full((N, Hq, D), np.nan)
    lse = np.full((N, Hq), np.nan)
    for b in range(len(lens)):
        n = starts[b + 1] - starts[b]
        if n == 0:
            continue
        K, V = gather(Kc, pages[b], lens[b]), gather(Vc, pages[b], lens[b])
        for i in range(starts[b], starts[b + 1]):
            seen = max(0, int(lens[b]) - (int(starts[b + 1]) - i) + 1)
            if seen == 0:
                O[i], M[i], lse[i] = 0.0, 0.0, -np.inf
                continue
            s = scale * np.einsum("hgd,htd->hgt", Q[i].reshape(Hk, Hq // Hk, D), K[:, :seen])
            m = s.max(-1, keepdims=True)
            p = np.exp(s - m)
            l = p.sum(-1, keepdims=True)
            O[i] = (p / l @ V[:, :seen]).reshape(Hq, D)
            M[i] = (p / l @ np.abs(V[:, :seen])).reshape(Hq, D)
            lse[i] = (m + np.log(l)).reshape(Hq)
    return O, lse, M
