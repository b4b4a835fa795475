"""Inputs and error bounds of the 4-bit cache's tests (test code; may use the
oracle)."""
from __future__ import annotations

import numpy as np
import torch

from attn_helpers import DEV, Batch, check_close
from helpers import U_F32, rel, ulp
from oracle import attn_oracle as A
from oracle import fp4_oracle as F
from oracle.ssn_oracle import f64
from paper_2607_13332_amd import inputs as I


def to_dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Fp4Batch(Batch):
    """Sequences over a paged 4-bit cache: codes of normal values where a
    sequence is, any bytes (NaN scales among them) everywhere else.  Kc and Vc
    are the values that the codes stand for."""

    def __init__(self, seqs, Hk, D, page, seed, **more):
        super().__init__(seqs, Hk, D, page, "f32", seed, **more)
        r = np.random.default_rng(seed + 1000)
        self.held = []
        for cache in (self.Kc, self.Vc):
            n = cache.shape[:3]
            codes = r.integers(0, 256, (*n, D // 2)).astype(np.uint8)
            scales = r.choice(np.array([255, 254, 0, 127], np.uint8), (*n, D // F.GROUP))
            for b in range(len(self.lens)):
                page_, off = self.slots(b)
                codes[page_, :, off], scales[page_, :, off] = F.quantise(cache[page_, :, off])
            self.held += [codes, scales]
        self.refresh()

    def refresh(self):
        """Kc and Vc from the codes and scales."""
        with np.errstate(over="ignore"):
            self.Kc = F.values(*self.held[:2]).astype(np.float32)
            self.Vc = F.values(*self.held[2:]).astype(np.float32)

    def device(self):
        """(Kc, Ks, Vc, Vs, pages, starts, lens) on the GPU."""
        return (*[to_dev(a) for a in self.held], to_dev(self.pages), to_dev(self.starts), to_dev(self.lens))


def attention_bound(ref, mag, q, kmax, vmax, D, scale, length, dtype):
    """Per-element bound of an attention output against the float64 oracle.

    Keys and values are exact in the matrix cores' operands.  A score is a
    float32 sum of D products, of 3 D where a float32 query is taken in three
    bf16 planes (which hold all its bits): off by (n + 4) u sum|q||k| scale, at
    most e = (n + 4) u |scale| |q|_1 kmax (u: unit roundoff of the sums, n: D or
    3 D), and by 2^-22 of itself through the change of base and the exponential,
    and 2^-21 absolute.  A probability is off by twice that (its own and the
    sum's), by 2^-8 where it is rounded to bf16 (8 significant bits, spaced 2^-7 at
    1, and half of that is the most; three planes keep a float32 one to 2^-24), and the sums over `length` keys by length u for each part.  All
    of it multiplies mag = sum p |v|.  Exponentials below the smallest normal
    number, 2^-126, may be flushed to zero: length 2^-126 vmax.  The output's own
    rounding is one ulp."""
    planes = 1 if dtype == "bf16" else 3
    reach = abs(scale) * np.abs(f64(q)).sum(-1, keepdims=True) * kmax
    e = (planes * D + 4) * U_F32 * reach + 2.0 ** -22 * reach + 2.0 ** -21
    p = 2.0 * np.expm1(e) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) + 2.0 * planes * length * U_F32
    return ulp(ref, dtype == "bf16") + p * mag + length * 2.0 ** -126 * vmax


def check_attention(bt, Hq, Hk, D, dtype, q, out, lse, scale=None):
    scale = D ** -0.5 if scale is None else scale
    O, L, M = A.paged_attention(q, bt.Kc, bt.Vc, bt.pages, bt.starts, bt.lens, scale)
    kmax, vmax = (max([np.abs(A.gather(c, bt.pages[b], t)).max(initial=0) for b, t in enumerate(bt.lens)])
                  for c in (bt.Kc, bt.Vc))
    inside = ~np.isnan(L[:, 0])
    assert (f64(out[~inside]) == 7).all()
    bound = attention_bound(O, M, q, kmax, vmax, D, scale, bt.max_len, dtype)
    check_close("O", out[inside], O[inside], bound[inside])
    # scores of ordinary size: a flat bar as well
    if inside.any() and scale == D ** -0.5 and np.abs(O[inside]).max(initial=0) > 0:
        assert rel(out[inside], O[inside]) <= (3e-3 if dtype == "bf16" else 3e-6)
    if lse is not None:
        assert (lse[~inside] == 7).all()
        reach = abs(scale) * np.abs(f64(q)).sum(-1) * kmax
        n = D if dtype == "bf16" else 3 * D
        check_close("lse", lse[inside], L[inside],
                    (2.0 ** -20 + (n + 8) * 2.0 ** -22 * reach + bt.max_len * 2.0 ** -23)[inside])


def normal(r, shape, dtype, scale=1.0):
    return I.store(scale * r.standard_normal(shape), dtype)
