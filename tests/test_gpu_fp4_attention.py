"""Attention over a 4-bit cache on the GPU against the float64 oracle, which
attends to the values that the codes stand for."""
import numpy as np
import pytest
import torch

from attn_helpers import DEV, TORCH, check_close, dev, packed_rows
from fp4_helpers import Fp4Batch, check_attention, normal, to_dev
from helpers import U_F32, ulp
from oracle import attn_oracle as A
from oracle import fp4_oracle as F
from oracle.ssn_oracle import f64
from paper_2607_13332_amd import inputs as I
from paper_2607_13332_amd import ssn

pytestmark = pytest.mark.gpu

BATCHES = {
    "one": [(1, 1)],
    "tokens": [(1, 5), (1, 64), (0, 0), (1, 65), (1, 1000), (0, 9), (1, 128)],
    "chunks": [(3, 3), (17, 40), (0, 7), (130, 130), (5, 700)],
    "mixed": [(1, 300), (200, 333), (1, 1), (1, 77), (64, 64)],
    "empty rows": [(2, 1), (1, 0), (5, 2), (1, 3)],
    "long": [(70, 2500), (1, 3001)],
    "long tokens": [(1, 2500), (1, 2501), (1, 31), (1, 0)],
}
HEADS = [(40, 8, 128), (16, 16, 64), (14, 2, 64), (7, 1, 128), (3, 1, 256), (6, 2, 96), (2, 1, 32), (4, 4, 160),
         (2, 1, 320), (32, 1, 128)]


def attend(bt, Hq, Hk, D, dtype, seed, split=True, q=None, with_lse=True, scale=None, strided=0):
    r = np.random.default_rng(seed)
    if q is None:
        q = normal(r, (bt.N, Hq, D), dtype, 1.5)
    ws = ssn.paged_attention_fp4_workspace(bt.N, len(bt.lens), Hq, Hk, D, bt.max_q, bt.max_len, DEV,
                                           dtype=TORCH[dtype]) if split else None
    if ws is not None:
        ws.fill_(255)                              # NaN in any type
    Q = packed_rows(q, dtype, ld_extra=2 * Hk * D + strided - 1) if strided else dev(q, dtype)
    out = torch.full((bt.N, Hq, D), 7.0, dtype=TORCH[dtype], device=DEV)
    lse = torch.full((bt.N, Hq), 7.0, dtype=torch.float32, device=DEV) if with_lse else None
    ssn.paged_attention_fp4(Q, *bt.device(), bt.max_q, bt.max_len, scale=scale, out=out, lse=lse, workspace=ws)
    return q, I.to_host(out), None if lse is None else lse.cpu().numpy()


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS)
def test_attention(dtype, heads, split):
    Hq, Hk, D = heads
    for n, (name, page) in enumerate([("one", 16), ("tokens", 16), ("chunks", 64), ("mixed", 7), ("empty rows", 1),
                                      ("long", 100), ("mixed", 128), ("long tokens", 64)]):
        if Hq * D > 2000 and name == "long" and not split:
            continue
        bt = Fp4Batch(BATCHES[name], Hk, D, page, 11 + n, first=n % 3, pad=n % 2)
        print(f"[case] paged_attention_fp4 {dtype} {heads} {name} page={page} split={split}", flush=True)
        # (strided: 1 on the 16-byte grid, 2 off it)
        q, out, lse = attend(bt, Hq, Hk, D, dtype, n, split, with_lse=n % 2 == 0, strided=(0, 1, 0, 2)[n % 4])
        check_attention(bt, Hq, Hk, D, dtype, q, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seqs", [[(1, 4000)], [(1, 9000), (1, 50)], [(300, 700)], [(20, 3000), (40, 41)]])
def test_repeated_calls_give_the_same_bits(dtype, seqs):
    bt = Fp4Batch(seqs, 2, 128, 64, 3)
    q, one, lse1 = attend(bt, 10, 2, 128, dtype, 1)
    _, two, lse2 = attend(bt, 10, 2, 128, dtype, 1, q=q)
    assert np.array_equal(one, two) and np.array_equal(lse1, lse2)
    check_attention(bt, 10, 2, 128, dtype, q, one, lse1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 96, 256])
@pytest.mark.parametrize("new,length,Hq", [(1, 600, 4), (9, 9, 4), (200, 200, 4), (140, 1500, 2), (3, 400, 10)])
def test_what_a_row_does_not_see_has_no_effect(dtype, D, new, length, Hq):
    """NaN in keys and values of later positions: rows before them keep their
    bits, and rows that see one are NaN where it is."""
    bt = Fp4Batch([(new, length)], 2, D, 16, 5)
    q, clean, _ = attend(bt, Hq, 2, D, dtype, 2)
    check_attention(bt, Hq, 2, D, dtype, q, clean, None)
    for at in {new - 1, new // 2, min(1, new - 1)}:
        bad = Fp4Batch([(new, length)], 2, D, 16, 5)
        page, off = bad.slots(0)
        for j in range(length - new + at, length):
            bad.held[3][page[j], :, off[j], j % (D // 32)] = 255
            if j % 2:
                bad.held[1][page[j], :, off[j]] = 255
        _, out, _ = attend(bad, Hq, 2, D, dtype, 2, q=q)
        assert np.array_equal(out[:at], clean[:at]), at
        got = f64(out)
        # the value of the row's own position
        for i in range(at, new):
            g = (length - new + i) % (D // 32)
            assert np.isnan(got[i, :, 32 * g:32 * g + 32]).all(), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 4, 70])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_group_without_values_stays_in_its_place(dtype, new, D):
    """NaN scales of values in tiles that every row sees: 32 elements of the
    output, the others keep their bits.  Of a key: all of the head's."""
    Hq, Hk, length = 4, 2, 700
    bt = Fp4Batch([(new, length)], Hk, D, 16, 3)
    q, clean, _ = attend(bt, Hq, Hk, D, dtype, 2)
    page, off = bt.slots(0)
    bt.held[3][page[40], 1, off[40], 1] = 255
    _, out, _ = attend(bt, Hq, Hk, D, dtype, 2, q=q)
    got, want = f64(out), f64(clean)
    assert np.isnan(got[:, 2:, 32:64]).all()
    got[:, 2:, 32:64] = want[:, 2:, 32:64] = 0
    assert np.array_equal(got, want)
    bt.held[3][page[40], 1, off[40], 1] = 127
    bt.held[1][page[333], 0, off[333], 0] = 255
    _, out, _ = attend(bt, Hq, Hk, D, dtype, 2, q=q)
    assert np.isnan(f64(out)[:, :2]).all() and np.isfinite(f64(out)[:, 2:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 4, 70, 200])
@pytest.mark.parametrize("D", [64, 96, 128, 256, 320])
def test_values_past_the_range_of_bf16(dtype, new, D):
    """Scale bytes 253 and 254, which appends do not write: 6 2^126 and 2^128 are
    infinite.  A value like that makes one element of the rows that see it infinite,
    with its sign, or NaN, and may make the rest of its group NaN; other elements keep
    their bits, and so do rows before it."""
    Hq, Hk, length = 4, 2, 700
    bt = Fp4Batch([(new, length)], Hk, D, 16, 3)
    page, off = bt.slots(0)
    for at in (40, length - new, length - 1 - new // 2, length - 1):
        for c, byte, code in ((0, 253, 7), (17, 253, 15), (1, 254, 12), (31, 254, 4)):
            where = page[at], 1, off[at]
            bt.held[2][where][16:32] = 0
            bt.held[3][where][1] = byte
            q, clean, _ = attend(bt, Hq, Hk, D, dtype, 2)
            bt.held[2][where][16 + c // 2] = code << (4 * (c % 2))
            _, out, _ = attend(bt, Hq, Hk, D, dtype, 2, q=q)
            got, want = f64(out), np.array(f64(clean))
            see = slice(max(0, at - (length - new)), None), slice(2, None), 32 + c
            assert (np.isnan(got[see]) | (got[see] == (-np.inf if code > 7 else np.inf))).all(), (at, byte, code)
            got[see] = want[see] = 0
            nan = np.isnan(got)
            assert not nan[:see[0].start].any() and not nan[:, :2].any() and not np.delete(nan, np.s_[32:64], -1).any()
            assert np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want)), (at, byte, code)
            bt.held[2][where][16 + c // 2] = bt.held[3][where][1] = 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 4, 70])
@pytest.mark.parametrize("D", [64, 128, 256, 320])
def test_keys_past_the_range_of_bf16(dtype, new, D):
    """A key element of -2^128, under queries that are positive there: the heads that
    see it have no weight for it, as for a finite one of -2^74, or are NaN; the others
    keep their bits, and so do rows before it."""
    Hq, Hk, length = 4, 2, 700
    bt = Fp4Batch([(new, length)], Hk, D, 16, 3)
    page, off = bt.slots(0)
    q = np.array(f64(normal(np.random.default_rng(2), (new, Hq, D), dtype, 1.5)))
    q[:, :, 3] = np.abs(q[:, :, 3]) + 0.5
    q = I.store(q, dtype)
    for at in (40, length - 1 - new // 2):
        where = page[at], 1, off[at]
        bt.held[0][where][:] = 0
        bt.held[0][where][1] = 0xC0                    # element 3: -2
        bt.held[1][where][0] = 200
        _, clean, _ = attend(bt, Hq, Hk, D, dtype, 2, q=q)
        assert np.isfinite(f64(clean)).all()
        bt.held[1][where][0] = 254
        _, out, _ = attend(bt, Hq, Hk, D, dtype, 2, q=q)
        got, want = f64(out), np.array(f64(clean))
        see = slice(max(0, at - (length - new)), None), slice(2, None)
        bad = np.isnan(got[see]).all(-1)
        got[see][bad] = want[see][bad] = 0
        assert np.array_equal(got, want), at
        bt.held[1][where][0] = 200


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales_and_far_scores(dtype, scale):
    """Scores far apart (scale 4: hundreds), equal ones, a negative scale."""
    bt = Fp4Batch([(40, 300), (1, 2000)], 2, 128, 16, 8)
    q, out, lse = attend(bt, 4, 2, 128, dtype, 1, scale=scale)
    check_attention(bt, 4, 2, 128, dtype, q, out, lse, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 65])
def test_a_sequence_of_growing_scores(dtype, new):
    """Every 40 keys score higher than all before: the running maximum moves."""
    bt = Fp4Batch([(new, 1000), (1, 1000)], 1, 64, 16, 8)
    for b in range(2):
        page, off = bt.slots(b)
        ramp = np.zeros((1000, 1, 64))
        ramp[:, 0, 0] = np.repeat(1.5 ** np.arange(25) / 1000, 40)
        bt.held[0][page, :, off], bt.held[1][page, :, off] = F.quantise(ramp.astype(np.float32))
    bt.refresh()
    q = np.zeros((bt.N, 2, 64))
    q[:, :, 0] = 16.0
    q = I.store(q, dtype)
    _, out, lse = attend(bt, 2, 1, 64, dtype, 1, q=q)
    check_attention(bt, 2, 1, 64, dtype, q, out, lse)


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("dtype,Hq,Hk,D", [("bf16", 4, 2, 64), ("bf16", 10, 2, 128), ("bf16", 3, 1, 96),
                                           ("f32", 4, 2, 64), ("f32", 2, 1, 128), ("bf16", 2, 2, 256)])
def test_chunks_over_long_caches(dtype, Hq, Hk, D, split):
    """The widest row tiles, with and without key ranges, beside a single
    token and a prompt."""
    bt = Fp4Batch([(100, 8300), (1, 8200), (90, 100), (17, 17)], Hk, D, 48, 2, first=1, pad=2)
    q, out, lse = attend(bt, Hq, Hk, D, dtype, 4, split)
    check_attention(bt, Hq, Hk, D, dtype, q, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [65, 256, 300, 1000])
def test_many_sequences(dtype, B):
    r = np.random.default_rng(B)
    seqs = []
    for b in range(B):
        n = int(r.choice([0, 1, 1, 2, 5, 33, 70]))
        seqs.append((n, n + int(r.integers(0, 60)) if r.random() < 0.9 else 1))
    bt = Fp4Batch(seqs, 2, 64, 16, 3, first=5, pad=4)
    bt.max_q, bt.max_len = 200, 500
    q, out, lse = attend(bt, 8, 2, 64, dtype, 1)
    check_attention(bt, 8, 2, 64, dtype, q, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_staged_parts_with_an_odd_number_of_rows(dtype):
    """A chunk and single tokens, both in ranges."""
    bt = Fp4Batch([(517, 7000), (1, 7000), (1, 3)], 1, 128, 64, 2)
    q, out, lse = attend(bt, 7, 1, 128, dtype, 1)
    check_attention(bt, 7, 1, 128, dtype, q, out, lse)


@pytest.mark.parametrize("new", [1, 5])
@pytest.mark.parametrize("D", [64, 128, 256, 96])
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
    bt = Fp4Batch(seqs, Hk, D, 16, 7)
    r = np.random.default_rng(D + new)
    for b, (_, length) in enumerate(seqs):
        page, off = bt.slots(b)
        # the first `visible` keys have no weight, the others almost the same
        x = np.zeros((length, Hk, D))
        x[:, :, 0] = np.where(np.arange(length)[:, None] < visible, -192.0, r.uniform(-0.2, 0.2, (length, Hk)))
        bt.held[0][page, :, off], bt.held[1][page, :, off] = F.quantise(x.astype(np.float32))
        v = np.where((np.arange(length)[:, None, None] + np.arange(D)) % 2, 1.0, -1.0) * np.ones((1, Hk, 1))
        bt.held[2][page, :, off], bt.held[3][page, :, off] = F.quantise(v.astype(np.float32))
    bt.refresh()
    q = np.zeros((bt.N, Hq, D))
    q[:, :, 0] = 1.0
    q = I.store(q, "bf16")
    for split in (True, False):
        _, out, _ = attend(bt, Hq, Hk, D, "bf16", 0, split, q=q, scale=1.0)
        O, _, M = A.paged_attention(q, bt.Kc, bt.Vc, bt.pages, bt.starts, bt.lens, 1.0)
        assert np.abs(O).min() < 0.06
        check_close("O", out, O, ulp(O, True) + (2.0 ** -16 + 2.0 ** -20 + 32 * U_F32) * M)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 40])
def test_queries_that_are_not_finite(dtype, new):
    """A NaN or an infinity in one query: its own head's output, no other."""
    bt = Fp4Batch([(new, 100)], 1, 64, 16, 3)
    q, clean, _ = attend(bt, 4, 1, 64, dtype, 2)
    bad = np.array(f64(q))
    bad[0, 1, 5], bad[new - 1, 2, 9] = np.nan, np.inf
    _, out, _ = attend(bt, 4, 1, 64, dtype, 2, q=I.store(bad, dtype))
    got, want = f64(out), f64(clean)
    assert np.isnan(got[0, 1]).all() and np.isnan(got[new - 1, 2]).all()
    got[0, 1] = want[0, 1] = got[new - 1, 2] = want[new - 1, 2] = 0
    assert np.array_equal(got, want)


@pytest.mark.parametrize("new", [1, 33])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_near_the_limit(dtype, new):
    """2047 x 2^20 keys, every table entry the same page.  Keys are zero, so every
    probability is one, and values are zeros and ones: the sums over one of 256
    ranges (8.4 million keys) are whole numbers below 2^24, exact in float32.  Left
    are 256 additions and multiplications of the join, a division, and of the
    logarithm (21.5) some units of 2^-20."""
    page, width, D = 2 ** 20, 2047, 32
    length = width * page - 5
    r = np.random.default_rng(3)
    v = r.integers(0, 2, (page, D)).astype(np.float64)
    held = [to_dev(a[None, None]) for x in (np.zeros((page, D), np.float32), v.astype(np.float32))
            for a in F.quantise(x)]
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    ws = ssn.paged_attention_fp4_workspace(new, 1, 1, 1, D, new, length, DEV, dtype=TORCH[dtype])
    assert ws is not None
    q = dev(normal(r, (new, 1, D), dtype), dtype)
    out = torch.full((new, 1, D), 7e6, dtype=TORCH[dtype], device=DEV)
    lse = torch.full((new, 1), 7e6, dtype=torch.float32, device=DEV)
    print(f"[case] attention of {new} tokens over {length} keys", flush=True)
    ssn.paged_attention_fp4(q, *held, torch.zeros((1, width), dtype=torch.int32, device=DEV), i32([0, new]), i32([length]),
                            new, length, out=out, lse=lse, workspace=ws)
    # position t is key t mod 2^20; token i sees length - new + i + 1 of them
    seen = length - new + 1 + np.arange(new)
    ones = seen[:, None] // page * v.sum(0) + np.stack([v[:n % page].sum(0) for n in seen])
    ref = ones / seen[:, None]
    join = 2 * 256 * U_F32
    check_close("O", I.to_host(out)[:, 0], ref, ulp(ref, dtype == "bf16") + join * ref)
    check_close("lse", lse.cpu().numpy()[:, 0], np.log(seen), np.full(new, join + 2.0 ** -17))


def test_cache_past_two_gibi():
    """A cache of more than 2^31 codes, its last pages in use."""
    Hk, D, page = 8, 128, 64
    bt = Fp4Batch([(1, 200), (130, 150)], Hk, D, page, 3, extra_pages=1)
    npages = 2 ** 31 // (Hk * page * D // 2) + 40
    cache = []
    last = npages - bt.held[0].shape[0]
    for a in bt.held:
        c = torch.zeros((npages, *a.shape[1:]), dtype=torch.uint8, device=DEV)
        c[last:] = to_dev(a)
        cache.append(c)
    n = bt.held[0].shape[0]
    pages = np.where((bt.pages >= 0) & (bt.pages < n), bt.pages + last, bt.pages).astype(np.int32)
    q = normal(np.random.default_rng(0), (bt.N, 16, D), "bf16", 1.5)
    ws = ssn.paged_attention_fp4_workspace(bt.N, 2, 16, Hk, D, bt.max_q, bt.max_len, DEV)
    out = ssn.paged_attention_fp4(dev(q, "bf16"), *cache, to_dev(pages), to_dev(bt.starts), to_dev(bt.lens), bt.max_q,
                                  bt.max_len, workspace=ws)
    check_attention(bt, 16, Hk, D, "bf16", q, I.to_host(out), None)


def test_other_stream_and_no_sync():
    """On a side stream, ordered after the work that makes the inputs there."""
    bt = Fp4Batch([(1, 500), (60, 900)], 2, 128, 64, 5)
    q, ref, _ = attend(bt, 8, 2, 128, "bf16", 2, with_lse=False)
    *cache, pages, starts, lens = bt.device()
    ws = ssn.paged_attention_fp4_workspace(bt.N, 2, 8, 2, 128, bt.max_q, bt.max_len, DEV)
    Q = dev(q, "bf16")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        late = [torch.zeros_like(c) for c in cache]
        out = torch.empty_like(Q)
        torch.cuda._sleep(2_000_000)
        for a, b in zip(late, cache):
            a.copy_(b)
        ssn.paged_attention_fp4(Q, *late, pages, starts, lens, bt.max_q, bt.max_len, out=out, workspace=ws)
    st.synchronize()
    assert np.array_equal(I.to_host(out), ref)


def test_graph_of_a_decode_step_follows_its_lengths():
    """One captured step (append, attention, read-back) replayed while the
    sequences grow, eager work between the replays, each replay against the
    eager calls."""
    Hq, Hk, D, page, T = 8, 2, 128, 16, 90
    r = np.random.default_rng(3)
    bt = Fp4Batch([(1, 70), (1, 3), (1, 31)], Hk, D, page, 5, extra_width=4, extra_pages=20)
    used = set(int(p) for b in range(3) for p in bt.slots(b)[0])
    free = [p for p in range(bt.Kc.shape[0]) if p not in used]
    for b in range(3):
        for j in range(-(-int(bt.lens[b]) // page), bt.pages.shape[1]):
            if free:
                bt.pages[b, j] = free.pop()
    *cache, pages, starts, lens = bt.device()
    table = ssn.rope_table(T + 100, D, 5e5, device=DEV)
    w = torch.ones(D, dtype=torch.bfloat16, device=DEV)
    qkv = torch.zeros((3, (Hq + 2 * Hk) * D), dtype=torch.bfloat16, device=DEV)
    heads = qkv.view(3, Hq + 2 * Hk, D)
    Qr, O = (torch.zeros((3, Hq, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    K, V = (torch.zeros((3, Hk, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ws = ssn.paged_attention_fp4_workspace(3, 3, Hq, Hk, D, 1, T, DEV)

    def step(Qr, O, K, V, cache):
        ssn.kv_append_fp4(heads[:, Hq:Hq + Hk], heads[:, Hq + Hk:], *cache, pages, starts, lens, Q=heads[:, :Hq],
                          table=table, wq=w, wk=w, Qout=Qr)
        ssn.paged_attention_fp4(Qr, *cache, pages, starts, lens, 1, T, out=O, workspace=ws)
        ssn.kv_read_fp4(*cache, pages, starts, lens, 3, Kout=K, Vout=V)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step(Qr, O, K, V, cache)
    torch.cuda.current_stream().wait_stream(st)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(Qr, O, K, V, cache)
    for n in range(6):
        qkv.copy_(dev(normal(r, tuple(qkv.shape), "bf16"), "bf16"))
        lens += 1
        c2, mine = [c.clone() for c in cache], [torch.zeros_like(x) for x in (Qr, O, K, V)]
        g.replay()
        step(*mine, c2)
        torch.cuda.synchronize()
        for a, b in zip((Qr, O, K, V, *cache), (*mine, *c2)):
            assert torch.equal(a, b), n
        assert torch.isfinite(O.float()).all() and (O != 0).any()
    assert int(lens[0]) == 76


def test_bounds_below_the_contents_stay_in_bounds():
    """max_q and max_len below what the batch holds, row ranges past N, page
    numbers out of range: unspecified results, no access outside the buffers
    (guard rows around the output keep their values)."""
    bt = Fp4Batch([(5, 300), (40, 90), (1, 1000)], 2, 64, 16, 3)
    *cache, pages, starts, lens = bt.device()
    Q = torch.zeros((bt.N, 8, 64), dtype=torch.bfloat16, device=DEV)
    guard = torch.full((bt.N + 64, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    out = guard[32:32 + bt.N]
    for max_q, max_len in [(1, 10), (3, 1000), (40, 100)]:
        ws = ssn.paged_attention_fp4_workspace(bt.N, 3, 8, 2, 64, max_q, max_len, DEV)
        ssn.paged_attention_fp4(Q, *cache, pages, starts, lens, max_q, max_len, out=out, workspace=ws)
    far = torch.tensor([0, 10 ** 6, -5, 10 ** 9], dtype=torch.int32, device=DEV)
    ssn.paged_attention_fp4(Q, *cache, pages, far, lens * 1000, 40, 10 ** 6, out=out)
    ssn.paged_attention_fp4(Q, *cache, torch.full_like(pages, -7), starts, lens, 40, 1000, out=out)
    torch.cuda.synchronize()
    assert (guard[:32] == 7).all() and (guard[32 + bt.N:] == 7).all()


def test_many_sequences_without_new_tokens():
    """200000 sequences of which four have new tokens, under bounds that allow
    128 ranges of keys."""
    B, page, Hq, Hk, D, max_len = 200_000, 64, 4, 1, 64, 32768
    few = Fp4Batch([(64, 9000), (1, 20000), (3, 3), (50, 700)], Hk, D, page, 4, pad=2)
    at = [0, 17, 123_456, B - 1]
    pages = np.full((B, max_len // page), -1, np.int32)
    lens = np.full(B, 5, np.int32)
    new = np.zeros(B, np.int64)
    for b, n in enumerate(at):
        pages[n, :few.pages.shape[1]] = few.pages[b]
        lens[n], new[n] = few.lens[b], few.new[b]
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = normal(np.random.default_rng(1), (few.N, Hq, D), "bf16", 1.5)
    ws = ssn.paged_attention_fp4_workspace(few.N, B, Hq, Hk, D, few.max_q, max_len, DEV)
    out = torch.full((few.N, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    print(f"[case] attention, {B} sequences", flush=True)
    ssn.paged_attention_fp4(dev(q, "bf16"), *few.device()[:4], to_dev(pages), to_dev(starts), to_dev(lens), few.max_q,
                            max_len, out=out, workspace=ws)
    check_attention(few, Hq, Hk, D, "bf16", q, I.to_host(out), None)


def test_a_quantised_stage_against_a_bf16_one():
    """Appended to both caches: attention over the 4-bit one is attention over a
    bf16 cache that holds what was read back, to the last bit but one."""
    Hq, Hk, D, page = 10, 2, 128, 16
    bt = Fp4Batch([(40, 40), (1, 1), (300, 300)], Hk, D, page, 3)
    r = np.random.default_rng(0)
    k, v, q = (dev(normal(r, (bt.N, h, D), "bf16"), "bf16") for h in (Hk, Hk, Hq))
    *cache, pages, starts, lens = bt.device()
    table = ssn.rope_table(400, D, 5e5, device=DEV)
    Q = ssn.kv_append_fp4(k, v, *cache, pages, starts, lens, Q=q, table=table)
    K, V = ssn.kv_read_fp4(*cache, pages, starts, lens, bt.N)
    Kc, Vc = (torch.zeros((bt.Kc.shape[0], Hk, page, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ssn.kv_append(K, V, Kc, Vc, pages, starts, lens, eps=None)
    O4 = ssn.paged_attention_fp4(Q, *cache, pages, starts, lens, bt.max_q, bt.max_len)
    O = ssn.paged_attention(Q, Kc, Vc, pages, starts, lens, bt.max_q, bt.max_len)
    # the flat bar of each against the exact value
    assert ((O4.float() - O.float()).norm() / O.float().norm()).item() <= 2 * 3e-3


def test_wrappers_refuse():
    bt = Fp4Batch([(1, 20), (3, 9)], 2, 64, 16, 3)
    Kc, Ks, Vc, Vs, pages, starts, lens = bt.device()
    Q = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device=DEV)
    att = lambda *a, **k: ssn.paged_attention_fp4(*a, pages, starts, lens, 3, 20, **k)  # noqa: E731
    with pytest.raises(TypeError, match="Kc must be torch.uint8"):
        att(Q, Kc.float(), Ks, Vc, Vs)
    with pytest.raises(ValueError, match="shape mismatch"):
        att(Q, Kc, Vs[..., :1], Vc, Vs)
    with pytest.raises(ValueError, match="shape mismatch"):         # heads of another size
        att(torch.zeros((4, 4, 128), dtype=torch.bfloat16, device=DEV), Kc, Ks, Vc, Vs)
    with pytest.raises(ValueError, match="out has shape"):
        att(Q, Kc, Ks, Vc, Vs, out=Q[:3])
    with pytest.raises(ValueError, match="different devices"):
        att(Q, Kc, Ks, Vc.cpu(), Vs)
    with pytest.raises(ssn.SSNError, match="status 7"):
        att(Q, Kc, Ks, Vc, Vs, out=Q)
    with pytest.raises(ssn.SSNError, match="status 2"):             # 3 query heads over 2 key heads
        att(Q[:, :3].contiguous(), Kc, Ks, Vc, Vs)
    with pytest.raises(ValueError, match="lse has shape"):
        att(Q, Kc, Ks, Vc, Vs, lse=torch.zeros((4, 3), device=DEV))
    with pytest.raises(TypeError, match="unsupported storage dtype"):
        att(Q.half(), Kc, Ks, Vc, Vs)
