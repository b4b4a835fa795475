"""The example of a stage's attention sublayer runs over a 4-bit cache, and a
sequence moves to another cache as it is."""
import pytest
import torch

from attn_helpers import DEV
from fp4_helpers import Fp4Batch, to_dev
from paper_2607_13332_amd import ssn
from test_gpu_stage_attention import _example

pytestmark = pytest.mark.gpu


def test_serving_runs():
    steps, whole = _example().serve(tokens=5, prompts=(70, 1, 300), chunk=64, fp4=True)
    assert steps.shape == whole.shape and torch.isfinite(steps).all() and torch.isfinite(whole).all()
    assert (steps != 0).any()


@pytest.mark.parametrize("length", [1, 300])
def test_a_sequence_moves(length):
    bt = Fp4Batch([(0, 40), (1, length)], 2, 128, 16, 5)
    *cache, pages, starts, lens = bt.device()
    other, numbers = _example().move(cache, pages[1:].contiguous(), length, 48)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    rows = (i32([0, length]), i32([length]))
    before = ssn.kv_read_fp4(*cache, pages[1:].contiguous(), *rows, length, dtype=torch.float32)
    after = ssn.kv_read_fp4(*other, numbers, *rows, length, dtype=torch.float32)
    page, off = bt.slots(1)
    for a, b, c in zip(before, after, (bt.Kc, bt.Vc)):
        assert torch.equal(a, b) and torch.equal(a, to_dev(c[page, :, off]))
