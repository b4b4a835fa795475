"""A stage that serves from a 4-bit cache: what it gives in chunks and token by
token against whole prompts and against the bf16 cache, and attention over the
4-bit cache against attention over a bf16 cache of the same values."""
import numpy as np
import pytest
import torch

from attn_helpers import DEV, attention_bound as stored_bound, check_close, dev
from fp4_helpers import Fp4Batch, attention_bound, normal
from oracle import attn_oracle as A
from oracle.ssn_oracle import f64
from paper_2607_13332_amd import inputs as I
from paper_2607_13332_amd import ssn
from test_gpu_stage_attention import _example

pytestmark = pytest.mark.gpu


def _attended(fp4):
    """What attention adds to the coordinates of each prompt's last token: fed in
    chunks and token by token, and fed whole (the coordinates that came in are
    three times as large)."""
    mod, seen = _example(), []
    serve = mod.Stage.serve
    mod.Stage.serve = lambda self, Z, *a: (seen.append(Z), serve(self, Z, *a))[1]
    steps, whole = mod.serve(tokens=5, prompts=(70, 1, 300), chunk=64, fp4=fp4)
    # the last call has the whole prompts, one after the other
    came = seen[-1][torch.tensor([75, 75 + 6, 75 + 6 + 305], device=DEV) - 1].float()
    assert seen[-1].shape[0] == 386
    return steps.float() - came, whole.float() - came


def test_serving_gives_what_whole_prompts_give():
    """Products of other tile shapes sum 1024 terms in another order: errors of
    about sqrt(1024) 2^-24 of sum |terms|, 25 times a result's size, carry one in
    40 of the bf16 activations over to a neighbour, 2^-7 away at most.  Such an
    element x passes a border between codes with a probability of 2^-7 |x| / s, s
    the distance of the levels, and moves by s: of its group's mean square 2^-7
    mean(|x| s) / mean(x^2), below 0.7 / 128, so sqrt(0.7 / 128 / 40) = 0.012 of
    keys and values.  Values carry that to the output as it is, keys through
    scores that are off by 0.012 of a unit normal: 0.017, twice the flat bar
    of attention (3e-3) more, and at most 0.004 for the sum with the residual stream,
    which is rounded to bf16 (2^-8 of it at most, of which a quarter falls into the 64
    of 1024 dimensions, against a third of its size)."""
    steps, whole = _attended(True)
    assert ((steps - whole).norm() / whole.norm()).item() <= 0.027


def test_serving_is_near_the_bf16_cache():
    """Normal values come back 11 % off: 0.11 of an output through the values, as
    much through scores that are off by 0.11 of a unit normal, 0.16 together.  A
    prompt's 64 coordinates scatter about that by a tenth of it; half as much
    again is the bar."""
    for a, b in zip(_attended(True), _attended(False)):
        assert ((a - b).norm(dim=-1) / b.norm(dim=-1)).max().item() <= 0.24


@pytest.mark.parametrize("seqs", [[(1, 700), (1, 33)], [(300, 300)], [(40, 40), (1, 1), (300, 300), (70, 1500)]])
def test_attention_is_that_over_a_bf16_cache_of_the_same_values(seqs):
    """Element by element, each within its bound of the exact value."""
    Hq, Hk, D, page = 10, 2, 128, 16
    bt = Fp4Batch(seqs, Hk, D, page, 3)
    q = normal(np.random.default_rng(0), (bt.N, Hq, D), "bf16", 1.5)
    *cache, pages, starts, lens = bt.device()
    # whole sequences as they are held
    rows = (torch.cat([lens.new_zeros(1), lens.cumsum(0).int()]), lens)
    K, V = ssn.kv_read_fp4(*cache, pages, *rows, int(rows[0][-1]))
    Kc, Vc = (torch.zeros((bt.Kc.shape[0], Hk, page, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ssn.kv_append(K, V, Kc, Vc, pages, *rows, eps=None)
    args = (pages, starts, lens, bt.max_q, bt.max_len)
    Q = dev(q, "bf16")
    O4, O = ssn.paged_attention_fp4(Q, *cache, *args), ssn.paged_attention(Q, Kc, Vc, *args)
    ref, _, mag = A.paged_attention(q, bt.Kc, bt.Vc, bt.pages, bt.starts, bt.lens, D ** -0.5)
    kmax, vmax = (max(np.abs(A.gather(c, bt.pages[b], t)).max() for b, t in enumerate(bt.lens)) for c in (bt.Kc, bt.Vc))
    b4 = attention_bound(ref, mag, q, kmax, vmax, D, D ** -0.5, bt.max_len, "bf16")
    # (2^-8 of a probability where it is rounded to bf16)
    b = stored_bound(ref, mag, q, kmax, D, D ** -0.5, bt.max_len, "bf16") + 2.0 ** -9 * mag
    check_close("O", I.to_host(O4), f64(I.to_host(O)), b4 + b)
