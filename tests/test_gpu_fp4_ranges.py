"""Attention over a 4-bit cache of very large and very small values."""
import numpy as np
import pytest

from fp4_helpers import Fp4Batch, check_attention
from test_gpu_fp4_attention import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hk,D", [(4, 2, 64), (10, 2, 128), (3, 1, 256), (2, 1, 320)])
@pytest.mark.parametrize("by", [105, -60])
def test_values_of_any_size(dtype, Hq, Hk, D, by):
    """Sums over at most 1024 keys are finite below 2^118 / 1024 = 2^108; normal
    values are below 8, and times 2^105 below that."""
    bt = Fp4Batch([(1, 1000), (200, 700), (3, 90)], Hk, D, 16, 3)
    for b in range(3):
        page, off = bt.slots(b)
        bt.held[3][page, :, off] += np.int8(by).astype(np.uint8)
    bt.refresh()
    assert max(np.abs(bt.Vc[bt.slots(b)[0], :, bt.slots(b)[1]]).max() for b in range(3)) < 2.0 ** (3 + by)
    print(f"[case] paged_attention_fp4 {dtype} {Hq}/{Hk}x{D}, values times 2^{by}", flush=True)
    q, out, lse = attend(bt, Hq, Hk, D, dtype, 1)
    check_attention(bt, Hq, Hk, D, dtype, q, out, lse)
    assert np.isfinite(lse).all()
