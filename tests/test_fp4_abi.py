"""CPU checks of the 4-bit cache's C ABI: bad arguments are refused on the host
before any HIP call (the fake addresses are never dereferenced), and the
validation is clean under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import shutil
import subprocess

import pytest
import torch

from test_attn_abi import (ERR_ALIAS, ERR_ALIGN, ERR_DTYPE, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, OK, ROOT, Call, lib)

__all__ = ["lib"]

A, B, C, D, E, F, G, H, J, K, L, M, N, P = ((0x7F00 + i) << 32 for i in range(14))
CODES, SCALES = 50 * 16 * 2 * 32, 50 * 16 * 2 * 2


def test_kv_append_fp4(lib):
    c = Call(lib.ssn_kv_append_fp4, dtype=1, N=10, B=3, Hq=4, Hk=2, D=64, R=64, P=100, style=0, eps=1e-6, Q=A, ldq=512,
             K=A + 512, ldk=512, V=A + 768, ldv=512, wq=B, wk=C, table=D, Kc=E, Ks=F, Vc=G, Vs=H, npages=50,
             page_size=16, pages=J, width=7, starts=K, lens=L, Qout=M, ldqo=256, stream=None)
    assert c.get(dtype=3) == ERR_DTYPE
    assert c.get(N=0, K=None, pages=None) == OK and c.get(B=0, K=None, starts=None) == OK
    for bad in [dict(N=-1), dict(B=-1), dict(B=1 << 20), dict(Hk=0), dict(npages=0), dict(page_size=0), dict(width=0),
                dict(width=1 << 28), dict(npages=1 << 28), dict(page_size=1 << 30), dict(ldv=127), dict(R=65),
                dict(eps=-1.0), dict(N=1 << 31), dict(D=80, ldq=1000, ldk=1000, ldv=1000, ldqo=1000),
                dict(D=48, R=48), dict(D=16, R=16), dict(D=0, R=0)]:
        assert c.get(**bad) == ERR_SHAPE, bad
    assert c.get(D=1056, ldq=9999, ldk=9999, ldv=9999, ldqo=9999) == ERR_UNSUPPORTED
    for name in ("Q", "K", "V", "table", "Kc", "Ks", "Vc", "Vs", "pages", "starts", "lens", "Qout"):
        assert c.get(**{name: None}) == ERR_NULL, name
    for name in ("Q", "K", "V", "Qout", "pages", "starts", "lens", "table"):
        assert c.get(**{name: c.args[name] + 1}) == ERR_ALIGN, name
    for bad in [dict(Ks=E + CODES - 1), dict(Vc=E + CODES - 1), dict(Vs=F + SCALES - 1), dict(Vs=F), dict(Kc=A),
                dict(Ks=A + 100), dict(Qout=E), dict(Qout=A), dict(Kc=J), dict(Vs=L), dict(Kc=D), dict(Vc=G, Kc=G)]:
        assert c.get(**bad) == ERR_ALIAS, bad


def test_kv_read_fp4(lib):
    c = Call(lib.ssn_kv_read_fp4, dtype=1, N=10, B=3, Hk=2, D=64, Kc=E, Ks=F, Vc=G, Vs=H, npages=50, page_size=16,
             pages=J, width=7, starts=K, lens=L, K=A, ldk=256, V=A + 256, ldv=256, stream=None)
    assert c.get(dtype=3) == ERR_DTYPE
    assert c.get(N=0, K=None, pages=None) == OK and c.get(B=0, K=None, starts=None) == OK
    for bad in [dict(N=-1), dict(B=-1), dict(B=1 << 20), dict(Hk=0), dict(npages=0), dict(page_size=0), dict(width=0),
                dict(width=1 << 28), dict(npages=1 << 28), dict(ldk=127), dict(ldv=100), dict(N=1 << 31), dict(D=80),
                dict(D=-32), dict(ldk=1 << 60)]:
        assert c.get(**bad) == ERR_SHAPE, bad
    assert c.get(D=1056, ldk=9999, ldv=9999) == ERR_UNSUPPORTED
    for name in ("Kc", "Ks", "Vc", "Vs", "pages", "starts", "lens", "K", "V"):
        assert c.get(**{name: None}) == ERR_NULL, name
    for name in ("K", "V", "pages", "starts", "lens"):
        assert c.get(**{name: c.args[name] + 1}) == ERR_ALIGN, name
    for bad in [dict(V=A + 128), dict(K=E + CODES - 2), dict(V=H), dict(K=J), dict(V=L + 8)]:
        assert c.get(**bad) == ERR_ALIAS, bad


def test_paged_attention_fp4(lib):
    c = Call(lib.ssn_paged_attention_fp4, dtype=1, N=10, B=3, Hq=4, Hk=2, D=64, max_q=4, max_len=100, scale=0.125,
             Q=A, ldq=512, Kc=B, Ks=C, Vc=D, Vs=E, npages=50, page_size=16, pages=F, width=7, starts=G, lens=H, O=J,
             ldo=256, lse=K, workspace=L, bytes=1 << 20, stream=None)
    assert c.get(dtype=2) == ERR_DTYPE
    assert c.get(N=0, Q=None, O=None) == OK and c.get(B=0, Q=None) == OK
    for bad in [dict(N=-1), dict(B=-1), dict(Hq=3), dict(Hq=0), dict(Hk=0), dict(D=0), dict(D=33), dict(D=80),
                dict(max_q=-1), dict(max_len=-1), dict(max_len=1 << 31), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(ldq=255), dict(ldo=100), dict(npages=0), dict(page_size=0),
                dict(width=0), dict(width=1 << 30), dict(npages=1 << 27), dict(N=1 << 30, Hq=4),
                dict(bytes=(1 << 64) - 1), dict(bytes=1 << 63)]:
        assert c.get(**bad) == ERR_SHAPE, bad
    assert c.get(D=1056, ldq=1 << 13, ldo=1 << 13) == ERR_UNSUPPORTED
    for name in ("Q", "Kc", "Ks", "Vc", "Vs", "pages", "starts", "lens", "O", "workspace"):
        assert c.get(**{name: None}) == ERR_NULL, name
    for name in ("Q", "pages", "starts", "lens", "O", "lse"):
        assert c.get(**{name: c.args[name] + 1}) == ERR_ALIGN, name
    assert c.get(workspace=L + 8) == ERR_ALIGN
    for bad in [dict(O=A), dict(O=A + 256, ldo=512), dict(O=B), dict(O=C), dict(lse=J), dict(lse=E),
                dict(workspace=K - (1 << 19)), dict(O=H), dict(workspace=D)]:
        assert c.get(**bad) == ERR_ALIAS, bad
    w = lib.ssn_paged_attention_fp4_workspace_bytes
    assert w(1, 0, 3, 4, 2, 64, 4, 100) == 0 and w(9, 10, 3, 4, 2, 64, 4, 100) == 0
    assert w(1, 10, 3, 3, 2, 64, 4, 100) == 0 and w(1, 10, 3, 4, 2, 4096, 4, 100) == 0
    assert w(1, 10, 3, 4, 2, 80, 4, 100) == 0 and w(1, 10, -3, 4, 2, 64, 4, 100) == 0


def test_wrappers_refuse_what_is_not_on_a_gpu():
    from paper_2607_13332_amd import ssn
    cache = ssn.fp4_cache(3, 2, 16, 64, "cpu") + ssn.fp4_cache(3, 2, 16, 64, "cpu")
    batch = (torch.zeros((1, 3), dtype=torch.int32), torch.tensor([0, 4], dtype=torch.int32),
             torch.tensor([4], dtype=torch.int32))
    x = torch.zeros((4, 2, 64))
    for call in (lambda: ssn.kv_append_fp4(x, x, *cache, *batch), lambda: ssn.kv_read_fp4(*cache, *batch, 4),
                 lambda: ssn.paged_attention_fp4(x, *cache, *batch, 4, 4)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    for bad in ((cache[0], cache[1][:2], *cache[2:]), (cache[0][..., :16], *cache[1:])):
        with pytest.raises(ValueError, match="shape mismatch"):
            ssn.paged_attention_fp4(x, *bad, *batch, 4, 4)
    with pytest.raises(ValueError, match="shape mismatch"):
        ssn.kv_append_fp4(x, x, *cache, *batch[:2], torch.tensor([4, 4], dtype=torch.int32))


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and the HIP headers")
def test_validation_is_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "fp4_asan")
    src, here = os.path.join(ROOT, "paper_2607_13332_amd", "csrc"), os.path.join(ROOT, "tests", "asan")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I" + os.path.join(ROOT, "include"), "-I" + src, "-x", "c++", os.path.join(src, "fp4_api.hip"),
           "-x", "none", os.path.join(here, "fp4_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "4-bit cache validation ok" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and the HIP headers")
def test_plans_fit_every_size(tmp_path):
    exe = str(tmp_path / "fp4_plan")
    cmd = ["g++", "-std=c++17", "-O2", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "paper_2607_13332_amd", "csrc"),
           os.path.join(ROOT, "tests", "asan", "fp4_plan_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "4-bit cache plans ok" in r.stdout


def test_workspace_sizes(lib):
    """Multiples of 16 bytes, and some where a long cache has few rows."""
    f = lib.ssn_paged_attention_fp4_workspace_bytes
    for dtype in (0, 1):
        for D in (32, 64, 96, 128, 256):
            for B, chunk, length in ((1, 1, 131072), (3, 1, 5000), (1, 512, 32768), (16, 200, 8000)):
                need = f(dtype, B - 1 + chunk, B, 8, 2, D, chunk, length)
                assert need % 16 == 0 and need < 1 << 33
            assert f(dtype, 1, 1, 8, 2, D, 1, 131072) > 0
