"""CPU check of the norm backward's grid, by the size of its workspace: a share
of both weight gradients (2 D float32) for every block of eight waves, and a
wave for every group of heads that a wave covers in one pass."""
import os

import pytest

WAVES = 8


@pytest.fixture(scope="module")
def lib():
    from paper_2607_13332_amd import ssn as mod
    if not os.path.exists(mod.LIB_PATH):
        from paper_2607_13332_amd import build
        build.build(verbose=False)
    return mod.lib()


@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_wave_for_every_pass(lib, dtype, size, D):
    # a lane holds 32 bytes of a head
    heads_per_wave = 64 * 32 // (D * size)
    for N in (1, 2, 3, 7, 100, 5000):
        for heads in [*range(1, 200), 8191, 8192, 8193, 9000, 16385, 32769, 40000]:
            for Hk in {0, 1, heads // 5, heads}:
                need = lib.ssn_qk_norm_rope_workspace_bytes(dtype, N, heads - Hk, Hk, D)
                blocks, rest = divmod(need, 2 * D * 4)
                assert rest == 0 and blocks >= 1
                passes = -(-heads // heads_per_wave)
                assert blocks * WAVES >= passes, (N, heads, Hk, blocks, passes)
