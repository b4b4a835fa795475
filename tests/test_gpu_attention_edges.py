"""The attention sublayer's calls at the edges of their contract."""
import numpy as np
import pytest
import torch

from attn_helpers import DEV, TORCH, Batch, attention_bound, check_close, dev
from helpers import U_F32, ulp
from oracle import attn_oracle as A
from paper_2607_13332_amd import inputs as I
from paper_2607_13332_amd import ssn

pytestmark = pytest.mark.gpu


def _nothing(*shape):
    """A tensor without elements whose strides are all zero (as numpy's are)."""
    return torch.empty(0, dtype=torch.bfloat16, device=DEV).as_strided(shape, (0, 0, 0))


def test_sides_without_heads_and_batches_without_rows():
    """Tensors without elements are taken whatever their strides are."""
    r = np.random.default_rng(0)
    x = I.store(r.standard_normal((3, 2, 64)), "bf16")
    X, none = dev(x, "bf16"), _nothing(3, 0, 64)
    Q, K = ssn.qk_norm_rope(X, none)
    K2 = ssn.qk_norm_rope(none, X)[1]
    ref = A.norm_rope(x)
    assert K.shape == (3, 0, 64) and torch.equal(Q, K2)
    assert np.abs(Q.double().cpu().numpy() - ref).max() <= 2.0 ** -8 * np.abs(ref).max()
    GQ, GK, _, _ = ssn.qk_norm_rope_backward(X, none, X, none)
    assert GK.shape == (3, 0, 64) and torch.equal(GQ, ssn.qk_norm_rope_backward(none, X, none, X)[1])
    bt = Batch([(0, 5)], 2, 64, 16, "bf16", 1)
    Kc, Vc, pages, starts, lens = bt.device()
    empty = _nothing(0, 2, 64)
    before = Kc.clone()
    assert ssn.kv_append(empty, empty, Kc, Vc, pages, starts, lens) is None
    assert torch.equal(Kc.view(torch.int16), before.view(torch.int16))
    assert ssn.paged_attention(_nothing(0, 4, 64), Kc, Vc, pages, starts, lens, 0, 5).shape == (0, 4, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_staged_parts_with_an_odd_number_of_rows(dtype):
    """A chunk and single tokens, both in ranges: 519 x 7 rows times 7 ranges of
    the tiles' results lie before those of the single tokens."""
    Hq, D = 7, 128
    bt = Batch([(517, 7000), (1, 7000), (1, 3)], 1, D, 64, dtype, 2)
    assert ssn.paged_attention_workspace_bytes(bt.N, 3, Hq, 1, D, bt.max_q, bt.max_len, TORCH[dtype]) > 0
    r = np.random.default_rng(1)
    q = I.store(1.5 * r.standard_normal((bt.N, Hq, D)), dtype)
    Kc, Vc, pages, starts, lens = bt.device()
    ws = ssn.paged_attention_workspace(bt.N, 3, Hq, 1, D, bt.max_q, bt.max_len, DEV, dtype=TORCH[dtype])
    ws.fill_(255)
    out = ssn.paged_attention(dev(q, dtype), Kc, Vc, pages, starts, lens, bt.max_q, bt.max_len, workspace=ws)
    O, _, M = A.paged_attention(q, bt.Kc, bt.Vc, bt.pages, bt.starts, bt.lens, D ** -0.5)
    kmax = max(np.abs(A.gather(bt.Kc, bt.pages[b], t)).max() for b, t in enumerate(bt.lens))
    check_close("O", I.to_host(out), O, attention_bound(O, M, q, kmax, D, D ** -0.5, bt.max_len, dtype))


@pytest.mark.parametrize("new", [1, 33])
def test_lengths_near_the_limit(new):
    """2047 x 2^20 keys, every table entry the same page.  Keys are zero, so every
    probability is one, and values are zeros and ones: the sums over one of 256
    ranges (8.4 million keys) are whole numbers below 2^24, exact in float32.  Left
    are 256 additions and multiplications of the join, a division, and of the
    logarithm (21.5) some units of 2^-20."""
    page, width, D = 2 ** 20, 2047, 8
    length = width * page - 5
    r = np.random.default_rng(3)
    v = r.integers(0, 2, (page, D)).astype(np.float64)
    cache = lambda a: dev(I.store(a[None, None], "bf16"), "bf16")  # noqa: E731
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    ws = ssn.paged_attention_workspace(new, 1, 1, 1, D, new, length, DEV)
    assert ws is not None
    q = dev(I.store(r.standard_normal((new, 1, D)), "bf16"), "bf16")
    out = torch.full((new, 1, D), 7e6, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((new, 1), 7e6, dtype=torch.float32, device=DEV)
    print(f"[case] attention of {new} tokens over {length} keys", flush=True)
    ssn.paged_attention(q, cache(np.zeros((page, D))), cache(v), torch.zeros((1, width), dtype=torch.int32, device=DEV),
                        i32([0, new]), i32([length]), new, length, out=out, lse=lse, workspace=ws)
    # position t is key t mod 2^20; token i sees length - new + i + 1 of them
    seen = length - new + 1 + np.arange(new)
    ones = seen[:, None] // page * v.sum(0) + np.stack([v[:n % page].sum(0) for n in seen])
    ref = ones / seen[:, None]
    join = 2 * 256 * U_F32
    check_close("O", I.to_host(out)[:, 0], ref, ulp(ref, True) + join * ref)
    check_close("lse", lse.cpu().numpy()[:, 0], np.log(seen), np.full(new, join + 2.0 ** -17))


def test_many_sequences_without_new_tokens():
    """200000 sequences of which four have new tokens, under bounds that allow
    128 ranges of keys: more blocks than a launch holds, if every sequence had
    them all."""
    B, page, Hq, Hk, D, max_len = 200_000, 64, 4, 1, 64, 32768
    few = Batch([(64, 9000), (1, 20000), (3, 3), (50, 700)], Hk, D, page, "bf16", 4, pad=2)
    at = [0, 17, 123_456, B - 1]
    pages = np.full((B, max_len // page), -1, np.int32)
    lens = np.full(B, 5, np.int32)
    new = np.zeros(B, np.int64)
    for b, n in enumerate(at):
        pages[n, :few.pages.shape[1]] = few.pages[b]
        lens[n], new[n] = few.lens[b], few.new[b]
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    r = np.random.default_rng(1)
    q = I.store(1.5 * r.standard_normal((few.N, Hq, D)), "bf16")
    Kc, Vc, *_ = few.device()
    i32 = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    ws = ssn.paged_attention_workspace(few.N, B, Hq, Hk, D, few.max_q, max_len, DEV)
    out = torch.full((few.N, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    print(f"[case] attention, {B} sequences", flush=True)
    ssn.paged_attention(dev(q, "bf16"), Kc, Vc, i32(pages), i32(starts), i32(lens), few.max_q, max_len, out=out,
                        workspace=ws)
    O, _, M = A.paged_attention(q, few.Kc, few.Vc, few.pages, few.starts, few.lens, D ** -0.5)
    kmax = max(np.abs(A.gather(few.Kc, few.pages[b], t)).max() for b, t in enumerate(few.lens))
    bound = attention_bound(O, M, q, kmax, D, D ** -0.5, few.max_len, "bf16")
    got, inside = I.to_host(out), slice(0, int(few.starts[-1]))
    check_close("O", got[inside], O[inside], bound[inside])
    assert (out[inside.stop:] == 7).all()


def test_rope_table_past_32_bits():
    """More than 2^31 pairs of a position (the table is 34 GB)."""
    R, theta = 2 ** 32 + 2, 1e4
    half = R // 2
    out = torch.full((2, R), 7.0, dtype=torch.float32, device=DEV)
    ssn.rope_table(2, R, theta, out=out)
    for i in (0, 1, half // 2, 2 ** 31 - 1, half - 1):
        a = theta ** (-2.0 * i / R)
        got = out[:, [i, half + i]].double().cpu().numpy()
        assert np.abs(got - [[1, 0], [np.cos(a), np.sin(a)]]).max() <= 2.0 ** -24 + 2.0 ** -50


@pytest.mark.parametrize("new", [1, 5])
@pytest.mark.parametrize("D", [64, 128, 256, 80])
@pytest.mark.parametrize("visible", [0, 500])
def test_probabilities_of_few_rows_keep_their_bits(D, new, visible):
    """bf16 rows of up to 32 of a key head: probabilities near each other under
    values of +-1, so that what is left of their sum is a few hundredths and a
    rounding of the probabilities to bf16 (2^-8 each) would show.

    Scores are single products (a query is a unit vector), exact in float32.  Left
    are 2^-16 of a probability (two bf16 parts), the exponential's 2^-20, sums of
    at most 14 terms that are not zero, and the output's rounding."""
    Hq, Hk = (6, 2) if new == 1 else (10, 2)
    if D == 256 and new > 1:
        Hq = 6
    seqs = [(new, visible + n) for n in (5, 6, 7, 9, 13, 14)]
    bt = Batch(seqs, Hk, D, 16, "bf16", 7)
    r = np.random.default_rng(D + new)
    for b, (_, length) in enumerate(seqs):
        page, off = bt.slots(b)
        # the first `visible` keys have no weight, the others almost the same
        x = np.zeros((length, Hk, D))
        x[:, :, 0] = np.where(np.arange(length)[:, None] < visible, -200.0, r.uniform(-0.2, 0.2, (length, Hk)))
        bt.Kc[page, :, off] = I.store(x, "bf16")
        v = np.where((np.arange(length)[:, None, None] + np.arange(D)) % 2, 1.0, -1.0) * np.ones((1, Hk, 1))
        bt.Vc[page, :, off] = I.store(v, "bf16")
    q = np.zeros((bt.N, Hq, D))
    q[:, :, 0] = 1.0
    q = I.store(q, "bf16")
    Kc, Vc, pages, starts, lens = bt.device()
    ws = ssn.paged_attention_workspace(bt.N, len(seqs), Hq, Hk, D, new, bt.max_len, DEV)
    for w in (ws, None):
        out = ssn.paged_attention(dev(q, "bf16"), Kc, Vc, pages, starts, lens, new, bt.max_len, scale=1.0, workspace=w)
        O, _, M = A.paged_attention(q, bt.Kc, bt.Vc, bt.pages, bt.starts, bt.lens, 1.0)
        assert np.abs(O).min() < 0.05
        check_close("O", I.to_host(out), O, ulp(O, True) + (2.0 ** -16 + 2.0 ** -20 + 32 * U_F32) * M)


@pytest.mark.parametrize("new", [1, 4])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("equal", [True, False])
def test_infinite_values_that_few_rows_see(D, new, equal):
    """An infinite value, positive or negative, in a tile that every row sees
    reaches its element with its sign, a NaN as one, and no other element."""
    Hq, Hk, length = 4, 2, 600
    bt = Batch([(new, length)], Hk, D, 16, "bf16", 3)
    r = np.random.default_rng(2)
    q = dev(I.store((0.0 if equal else 1.5) * r.standard_normal((new, Hq, D)), "bf16"), "bf16")
    Kc, Vc, pages, starts, lens = bt.device()
    ws = ssn.paged_attention_workspace(new, 1, Hq, Hk, D, new, length, DEV)
    for w in (ws, None):
        args = (pages, starts, lens, new, length)
        clean = ssn.paged_attention(q, Kc, Vc, *args, workspace=w).float()
        page, off = bt.slots(0)
        bad = Vc.clone()
        for t, e, x in [(3, 7, float("inf")), (40, 20, -float("inf")), (333, 40, float("nan")), (100, 41, 3e38)]:
            bad[int(page[t]), :, int(off[t]), e] = x
        got = ssn.paged_attention(q, Kc, bad, *args, workspace=w).float()
        assert (got[..., 7] == float("inf")).all() and (got[..., 20] == -float("inf")).all()
        assert torch.isnan(got[..., 40]).all() and torch.isfinite(got[..., 41]).all()
        keep = [e for e in range(D) if e not in (7, 20, 40, 41)]
        assert torch.equal(got[..., keep], clean[..., keep])
