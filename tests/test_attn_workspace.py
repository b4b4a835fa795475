"""CPU checks of the attention workspace's size."""
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2607_13332_amd import ssn as mod
    if not os.path.exists(mod.LIB_PATH):
        from paper_2607_13332_amd import build
        build.build(verbose=False)
    return mod.lib()


@pytest.mark.parametrize("dtype", [0, 1])
def test_every_part_of_the_workspace_is_16_byte_aligned(lib, dtype):
    """The parts follow each other, so each is a multiple of 16 bytes: batches
    of a chunk and single tokens, whose tiles have an odd number of rows."""
    staged = 0
    for Hq, Hk in [(7, 1), (3, 1), (5, 5), (40, 8)]:
        for D in (64, 80, 128, 256):
            for B, chunk in [(3, 517), (2, 101), (5, 64), (4, 1001)]:
                for max_len in (2000, 7000, 8191, 40000):
                    need = lib.ssn_paged_attention_workspace_bytes(dtype, B - 1 + chunk, B, Hq, Hk, D, chunk, max_len)
                    assert need % 16 == 0, (Hq, Hk, D, B, chunk, max_len)
                    staged += need > 0
    assert staged > 100
