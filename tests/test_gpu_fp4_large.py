"""Appends to the 4-bit cache and reading it back, in batches large enough that a
wave takes several tokens at a time and goes on to more: every byte of the caches
and every element read back, against the definition in float64."""
import pytest
import torch

from attn_helpers import DEV, TORCH
from oracle import fp4_oracle as F
from paper_2607_13332_amd import ssn

pytestmark = pytest.mark.gpu

MANY = 2 ** 23            # elements of keys from which on a wave takes several tokens
WAVES = 32768             # of one launch
LEVELS = torch.tensor(F.LEVELS, dtype=torch.float64)


def _slabs(x, n=2 ** 23):
    step = max(1, n // max(1, x[0].numel()))
    return [slice(a, a + step) for a in range(0, x.shape[0], step)]


def _quantised(x):
    """Codes [.., D / 2] and scales [.., D / 32] of x [.., D], finite and not
    denormal: the smallest e with max < 7 2^e, the nearest of all levels, of two
    the even one."""
    codes = torch.empty((*x.shape[:-1], x.shape[-1] // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((*x.shape[:-1], x.shape[-1] // 32), dtype=torch.uint8, device=DEV)
    even = torch.arange(8, device=DEV) % 2 * 2.0 ** -30
    for s in _slabs(x):
        part = x[s].double().unflatten(-1, (-1, 32))
        m, E = torch.frexp(part.abs().amax(-1, keepdim=True))       # 8 m 2^(E - 3), 1/2 <= m < 1
        e = E - 3 + (m >= 0.875)
        v = torch.ldexp(part, -e)
        far = (v.abs()[..., None] - LEVELS.to(DEV)).abs_().add_(even)
        c = (far.argmin(-1) + 8 * torch.signbit(part)).to(torch.uint8).flatten(-2)
        codes[s] = c[..., 0::2] | (c[..., 1::2] << 4)
        scales[s] = (e + 127).squeeze(-1).to(torch.uint8)
    return codes, scales


def _values(codes, scales):
    """What codes and scales stand for, in float32 (exact)."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    level = torch.cat([LEVELS, -LEVELS]).float().to(DEV)
    return torch.ldexp(level[c].unflatten(-1, (-1, 32)), scales.int()[..., None] - 127).flatten(-2)


class Large:
    """Sequences (new tokens, length) over 4-bit caches of any bytes, pages handed
    out in no order, rows before the first sequence and padding behind the last."""

    def __init__(self, seqs, Hk, D, page, seed, first=3, pad=2):
        g = torch.Generator(device=DEV).manual_seed(seed)
        need = [-(-t // page) for _, t in seqs]
        order = torch.randperm(sum(need) + 2, generator=g, device=DEV).to(torch.int32)
        self.pages = torch.full((len(seqs), max(need) + 1), -1, dtype=torch.int32, device=DEV)
        starts, at = [first], 0
        for b, n in enumerate(need):
            self.pages[b, :n] = order[at:at + n]
            at += n
            starts.append(starts[-1] + seqs[b][0])
        self.N = starts[-1] + pad
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
        self.starts, self.lens = i32(starts), i32([t for _, t in seqs])
        shape = (sum(need) + 2, Hk, page)
        byte = lambda n: torch.randint(0, 256, (*shape, n), generator=g, device=DEV, dtype=torch.uint8)  # noqa: E731
        self.cache = [byte(D // 2), byte(D // 32), byte(D // 2), byte(D // 32)]
        # the rows that have a position, and their slots
        i = torch.arange(self.N, device=DEV)
        b = torch.searchsorted(self.starts, i.int(), right=True) - 1
        inside = (b >= 0) & (i < self.starts[-1])
        b = b.clamp(0, len(seqs) - 1)
        pos = self.lens[b] - (self.starts[b + 1] - i)
        self.has = inside & (pos >= 0)
        pos, b = pos[self.has], b[self.has]
        self.slots = self.pages[b, pos // page].long(), pos % page

    def batch(self):
        return self.pages, self.starts, self.lens


def _check(bt, cache, k, v, out):
    """Caches and what was read back, against the definition."""
    page, off = bt.slots
    for z, x in enumerate((k, v)):
        codes, scales = _quantised(x[bt.has])
        for name, got, was, new in (("codes", cache[2 * z], bt.cache[2 * z], codes),
                                    ("scales", cache[2 * z + 1], bt.cache[2 * z + 1], scales)):
            want = was.clone()
            want[page, :, off] = new
            assert torch.equal(got, want), ("KV"[z], name)
        if out is not None:
            assert torch.equal(out[z][bt.has].float(), _values(codes, scales)), "KV"[z]
            assert (out[z][~bt.has] == 7).all()


def _normal(g, shape, dtype):
    x = torch.empty(shape, dtype=TORCH[dtype], device=DEV)
    for s in _slabs(x):
        x[s] = torch.randn(x[s].shape, generator=g, device=DEV)
    return x


def _sizes(B, n, g):
    """Of B sequences of about n new tokens each: empty ones at the ends and
    between, single tokens, a few lengths below the new tokens."""
    seqs = [(0, 3)]
    for j, x in enumerate(torch.randint(1, 2 * n, (B - 2,), generator=g).tolist()):
        new = (x, x, 1, x, 0, x, x, 2)[j % 8]
        seqs.append((new, max(0, new + (0, 5, 40, -3)[j % 4])))
    return seqs + [(0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [1, 63, 64, 65, 300])
@pytest.mark.parametrize("Hk,D", [(8, 128), (16, 64), (8, 96)])
def test_several_tokens_to_a_wave(dtype, Hk, D, B):
    """On both sides of the 64 sequences that a wave holds in its lanes: a wave's
    tokens are of one sequence, or of several, or padding."""
    g = torch.Generator().manual_seed(B)
    n = 12_001
    bt = Large([(n, n + 7)] if B == 1 else _sizes(B, n // B * 2, g), Hk, D, 16, B)
    assert bt.N * Hk * D >= MANY
    g = torch.Generator(device=DEV).manual_seed(B + 1)
    k, v = (_normal(g, (bt.N, Hk, D), dtype) for _ in range(2))
    cache = [c.clone() for c in bt.cache]
    print(f"[case] kv_append_fp4 and kv_read_fp4 {dtype} {Hk} heads of {D}, {B} sequences, {bt.N} rows", flush=True)
    ssn.kv_append_fp4(k, v, *cache, *bt.batch(), eps=None)
    out = [torch.full((bt.N, Hk, D), 7.0, dtype=TORCH[dtype], device=DEV) for _ in range(2)]
    ssn.kv_read_fp4(*cache, *bt.batch(), bt.N, Kout=out[0], Vout=out[1])
    _check(bt, cache, k, v, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,D,N,B", [(8, 128, 65_611, 64), (8, 128, 65_611, 70), (2, 96, 262_209, 64)])
def test_a_wave_goes_on_to_more_tokens(dtype, Hk, D, N, B):
    """More tokens than all waves of a launch take at first: four each where they
    append, eight where they read back."""
    first = 8 * (WAVES // -(-2 * Hk * D // 8 // 64))
    g = torch.Generator().manual_seed(N + B)
    seqs = _sizes(B, N // B, g)
    left = N - sum(n for n, _ in seqs)
    seqs[B // 2] = (seqs[B // 2][0] + max(left, 0) + 1,) * 2
    bt = Large(seqs, Hk, D, 64, B)
    assert bt.N > first
    g = torch.Generator(device=DEV).manual_seed(B + 1)
    k, v = (_normal(g, (bt.N, Hk, D), dtype) for _ in range(2))
    cache = [c.clone() for c in bt.cache]
    print(f"[case] kv_append_fp4 and kv_read_fp4 {dtype} {Hk} heads of {D}, {B} sequences, {bt.N} rows", flush=True)
    ssn.kv_append_fp4(k, v, *cache, *bt.batch(), eps=None)
    out = [torch.full((bt.N, Hk, D), 7.0, dtype=TORCH[dtype], device=DEV) for _ in range(2)]
    ssn.kv_read_fp4(*cache, *bt.batch(), bt.N, Kout=out[0], Vout=out[1])
    _check(bt, cache, k, v, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hk,D,N,B", [(40, 8, 128, 5000, 64), (40, 8, 128, 5000, 66), (16, 16, 64, 11_000, 9),
                                         (4, 2, 256, 33_000, 64)])
def test_queries_beside_more_tokens_than_waves(dtype, Hq, Hk, D, N, B):
    """The append with queries, more tokens than waves.  As they are: every byte.
    Normed and rotated: the bytes of calls of parts, each with a wave for every
    token."""
    per_wave = 64 * 2 * (8 if dtype == "bf16" else 4) // D
    slots = WAVES // -(-(Hq + 2 * Hk) // per_wave)
    g = torch.Generator().manual_seed(B)
    seqs = _sizes(B, N // B, g)
    left = N - sum(n for n, _ in seqs)
    seqs[B // 2] = (seqs[B // 2][0] + max(left, 0) + 1,) * 2
    bt = Large(seqs, Hk, D, 16, B)
    assert bt.N > slots
    g = torch.Generator(device=DEV).manual_seed(B + 1)
    q, k, v = (_normal(g, (bt.N, h, D), dtype) for h in (Hq, Hk, Hk))
    print(f"[case] kv_append_fp4 {dtype} {Hq} / {Hk} heads of {D}, {B} sequences, {bt.N} rows, {slots} waves a head", flush=True)
    cache = [c.clone() for c in bt.cache]
    Q = torch.full_like(q, 7.0)
    ssn.kv_append_fp4(k, v, *cache, *bt.batch(), Q=q, Qout=Q, eps=None)
    _check(bt, cache, k, v, None)
    assert torch.equal(Q[bt.has], q[bt.has]) and (Q[~bt.has] == 7).all()

    table = ssn.rope_table(int(bt.lens.max()), D, 5e5, device=DEV)
    w = [(1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(TORCH[dtype]) for _ in range(2)]
    whole, parts = [c.clone() for c in bt.cache], [c.clone() for c in bt.cache]
    Qp = torch.full_like(q, 7.0)
    Q.fill_(7)
    more = dict(table=table, wq=w[0], wk=w[1], eps=1e-6)
    ssn.kv_append_fp4(k, v, *whole, *bt.batch(), Q=q, Qout=Q, **more)
    for s in range(0, bt.N, slots // 2):
        e = min(s + slots // 2, bt.N)
        # of every sequence the rows in [s, e), at their positions
        starts = (bt.starts.clamp(s, e) - s).int()
        lens = bt.lens - (bt.starts[1:] - bt.starts[1:].clamp(s, e))
        ssn.kv_append_fp4(k[s:e], v[s:e], *parts, bt.pages, starts, lens.int(), Q=q[s:e], Qout=Qp[s:e], **more)
    for a, b in zip(whole, parts):
        assert torch.equal(a, b)
    assert torch.equal(Q, Qp) and (Q[~bt.has] == 7).all()
    # and values as they are
    page, off = bt.slots
    codes, scales = _quantised(v[bt.has])
    assert torch.equal(whole[2][page, :, off], codes) and torch.equal(whole[3][page, :, off], scales)
