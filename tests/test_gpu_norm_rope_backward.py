"""Gradients of the norms of heads where lanes or waves of the kernel have no
head, or more heads than an ordinary call: against the float64 oracle."""
import numpy as np
import pytest
import torch

from attn_helpers import DEV, TORCH, check_close, dev, packed_rows
from helpers import elementwise_bound
from oracle import attn_oracle as A
from oracle.ssn_oracle import f64
from paper_2607_13332_amd import inputs as I
from paper_2607_13332_amd import ssn

pytestmark = pytest.mark.gpu


def _inputs(dtype, Hq, Hk, D, N, seed):
    r = np.random.default_rng(seed)
    normal = lambda *s: I.store(r.standard_normal(s), dtype)  # noqa: E731
    q, k, gq, gk = normal(N, Hq, D), normal(N, Hk, D), normal(N, Hq, D), normal(N, Hk, D)
    wq, wk = (I.store(1 + 0.2 * r.standard_normal(D), dtype) for _ in range(2))
    return q, k, gq, gk, wq, wk, r.integers(0, 50, N).astype(np.int32), A.rope_table(50, D, 5e5).astype(np.float32)


def _check(dtype, x, gy, w, pos, table, eps, style, got, got_w, chain):
    """`chain`: roundings of a weight gradient's sum, one after the other."""
    D = x.shape[-1]
    ref, ref_w = A.norm_rope_backward(x, gy, w, pos, table, eps, style)
    f, g = np.abs(f64(x)), np.abs(f64(gy))
    r = 1 / np.sqrt((f * f).mean(-1, keepdims=True) + eps)
    # a turned element is at most sqrt(2) times the larger of its pair
    turned = np.broadcast_to(np.sqrt(2) * g.max(-1, keepdims=True), g.shape)
    h, n = turned * np.abs(f64(w)), f * r
    mag = r * (h + n * (h * n).mean(-1, keepdims=True))
    check_close("dL/dx", I.to_host(got), ref, elementwise_bound(ref, mag, D // 2 + 12, False, dtype == "bf16"))
    # a term: the rotation, half of the sum of squares' roundings, a few products
    check_close("dL/dw", I.to_host(got_w), ref_w,
                elementwise_bound(ref_w, (turned * n).sum((0, 1)), D // 4 + 10 + chain, False, False))


@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("dtype,Hq,Hk,D", [("bf16", 3, 1, 128), ("bf16", 32, 4, 128), ("bf16", 4, 2, 64),
                                           ("bf16", 5, 1, 256), ("f32", 3, 1, 64), ("f32", 2, 1, 256),
                                           ("f32", 4, 1, 128), ("f32", 1, 6, 128)])
def test_weight_gradients_without_eps(dtype, Hq, Hk, D, odd, style):
    """eps = 0 and head counts that leave lanes of the last wave without a
    head; `odd` moves the rows off the 16-byte grid."""
    N = 21
    q, k, gq, gk, wq, wk, pos, table = _inputs(dtype, Hq, Hk, D, N, 5)
    rows = packed_rows(np.concatenate([q, k], 1), dtype, ld_extra=D + odd, before=odd)
    print(f"[case] norm backward, eps 0: {dtype} {Hq}/{Hk} x {D} odd={odd} {style}", flush=True)
    GQ, GK, Gwq, Gwk = ssn.qk_norm_rope_backward(
        rows[:, :Hq], rows[:, Hq:], dev(gq, dtype), dev(gk, dtype), torch.from_numpy(pos).to(DEV),
        torch.from_numpy(table).to(DEV), dev(wq, dtype), dev(wk, dtype), eps=0.0, style=style)
    # N tokens of at most Hq or Hk heads each, one after the other at worst
    _check(dtype, q, gq, wq, pos, table, 0.0, style, GQ, Gwq, N * Hq)
    _check(dtype, k, gk, wk, pos, table, 0.0, style, GK, Gwk, N * Hk)


@pytest.mark.parametrize("N,dtype,Hq,Hk,D", [(1, "f32", 16, 1, 256), (1, "f32", 16, 4, 256), (1, "f32", 40, 8, 256),
                                             (1, "f32", 17, 0, 256), (1, "f32", 0, 17, 256), (1, "bf16", 40, 8, 256),
                                             (1, "f32", 40, 8, 128), (2, "f32", 9000, 500, 256),
                                             (1, "bf16", 17000, 100, 256), (1, "f32", 17000, 100, 128)])
def test_every_head_of_a_few_tokens(N, dtype, Hq, Hk, D):
    """More heads than 16 waves hold, and more than the waves of 512 blocks:
    every head's gradient is written (the outputs hold something else before),
    and the weight gradients have all terms."""
    q, k, gq, gk, wq, wk, pos, table = _inputs(dtype, Hq, Hk, D, N, 6)
    print(f"[case] norm backward, many heads: {dtype} N={N} {Hq}/{Hk} x {D}", flush=True)
    GQ, GK = (torch.full((N, h, D), 7e6, dtype=TORCH[dtype], device=DEV) for h in (Hq, Hk))
    _, _, Gwq, Gwk = ssn.qk_norm_rope_backward(
        dev(q, dtype), dev(k, dtype), dev(gq, dtype), dev(gk, dtype), torch.from_numpy(pos).to(DEV),
        torch.from_numpy(table).to(DEV), dev(wq, dtype), dev(wk, dtype), GQin=GQ, GKin=GK)
    # a wave's heads and tokens, a block's waves, the blocks' shares 16 at a time
    if Hq:
        _check(dtype, q, gq, wq, pos, table, 1e-6, "halves", GQ, Gwq, 60 + N * Hq // 64)
    if Hk:
        _check(dtype, k, gk, wk, pos, table, 1e-6, "halves", GK, Gwk, 60 + N * (Hq + Hk) // 64)
