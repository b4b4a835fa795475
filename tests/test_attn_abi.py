"""CPU checks of the attention sublayer's C ABI: bad arguments are refused on
the host before any HIP call (the fake addresses are never dereferenced), and
the validation is clean under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, ERR_NULL, ERR_SHAPE, ERR_DTYPE, ERR_ALIGN, ERR_UNSUPPORTED, ERR_LAUNCH, ERR_ALIAS = range(8)

# fake, never dereferenced device addresses, far apart
A, B, C, D, E, F, G, H, J, K, L, M = ((0x7F00 + i) << 32 for i in range(12))


@pytest.fixture(scope="module")
def lib():
    from paper_2607_13332_amd import ssn as mod
    if not os.path.exists(mod.LIB_PATH):
        from paper_2607_13332_amd import build
        build.build(verbose=False)
    return mod.lib()


class Call:
    """A call with valid defaults, by argument name; get(name=value) is its
    status with that changed."""

    def __init__(self, fn, **args):
        self.fn, self.args = fn, args

    def get(self, **change):
        assert set(change) <= set(self.args), change
        return self.fn(*{**self.args, **change}.values())


def norm_call(lib, **over):
    return Call(lib.ssn_qk_norm_rope, dtype=1, N=10, Hq=4, Hk=2, D=64, R=64, P=100, style=0, eps=1e-6, Q=A, ldq=512,
                K=A + 512, ldk=512, wq=B, wk=C, pos=D, table=E, Qout=F, ldqo=256, Kout=G, ldko=128, stream=None)


def test_rope_table(lib):
    f = lib.ssn_rope_table
    assert f(0, 64, 1e4, None, None) == OK and f(10, 0, 1e4, None, None) == OK
    assert f(10, 64, 1e4, None, None) == ERR_NULL
    assert f(10, 64, 1e4, A + 2, None) == ERR_ALIGN
    for P, R, theta in [(-1, 64, 1e4), (10, 63, 1e4), (10, -2, 1e4), (10, 64, 0.0), (10, 64, -1.0),
                        (10, 64, float("nan")), (10, 64, float("inf")), (1 << 40, 64, 1e4)]:
        assert f(P, R, theta, A, None) == ERR_SHAPE


def test_norm_rope(lib):
    c = norm_call(lib)
    assert c.get(dtype=7) == ERR_DTYPE
    assert c.get(N=0, Q=None, K=None, Qout=None, Kout=None, wq=None, wk=None) == OK
    for bad in [dict(N=-1), dict(Hq=-1), dict(Hq=0, Hk=0), dict(D=0), dict(R=63), dict(R=66), dict(R=-2), dict(P=0),
                dict(style=2), dict(style=-1), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=-1.0),
                dict(ldq=255), dict(ldk=127), dict(ldqo=255), dict(ldko=127), dict(N=1 << 31), dict(ldq=1 << 60),
                dict(Hq=1 << 30)]:
        assert c.get(**bad) == ERR_SHAPE, bad
    assert c.get(D=1026, ldq=10000, ldk=10000, ldqo=10000, ldko=10000) == ERR_UNSUPPORTED
    for name in ("Q", "K", "pos", "table", "Qout", "Kout"):
        assert c.get(**{name: None}) == ERR_NULL, name
    for name in ("Q", "K", "Qout", "Kout", "wq", "wk"):
        assert c.get(**{name: c.args[name] + 1}) == ERR_ALIGN, name
    assert c.get(pos=D + 2) == ERR_ALIGN and c.get(table=E + 2) == ERR_ALIGN
    for bad in [dict(Qout=A), dict(Kout=A + 512 + 64), dict(Kout=F + 64), dict(Qout=E + 4), dict(Qout=D),
                dict(Kout=B), dict(Qout=A + 128, ldqo=512)]:
        assert c.get(**bad) == ERR_ALIAS, bad
    # one side alone: the other's pointers and strides are not looked at
    c0 = dict(Hk=0, K=None, Kout=A, wk=3, ldk=-5, ldko=-(1 << 62))
    assert c.get(**c0, Q=None) == ERR_NULL


def test_norm_rope_backward(lib):
    c = Call(lib.ssn_qk_norm_rope_backward, dtype=1, N=10, Hq=4, Hk=2, D=64, R=64, P=100, style=0, eps=1e-6, Q=A,
             ldq=512, K=A + 512, ldk=512, wq=B, wk=C, pos=D, table=E, GQ=F, ldgq=256, GK=G, ldgk=128, GQin=H,
             ldgqi=512, GKin=H + 512, ldgki=512, Gwq=J, Gwk=K, workspace=L, bytes=1 << 20, stream=None)
    need = lib.ssn_qk_norm_rope_workspace_bytes(1, 10, 4, 2, 64)
    assert 0 < need <= 1 << 20 and need % (2 * 64 * 4) == 0
    assert lib.ssn_qk_norm_rope_workspace_bytes(1, 0, 4, 2, 64) == 0
    assert lib.ssn_qk_norm_rope_workspace_bytes(5, 10, 4, 2, 64) == 0
    assert lib.ssn_qk_norm_rope_workspace_bytes(1, -3, 4, 2, 64) == 0
    assert lib.ssn_qk_norm_rope_workspace_bytes(1, 10, 4, 2, 1 << 40) == 0
    assert c.get(dtype=-1) == ERR_DTYPE
    assert c.get(N=0, Gwq=None, Gwk=None) == OK
    for bad in [dict(bytes=need - 1), dict(eps=-1.0), dict(eps=-1.0, wq=None, wk=None), dict(ldgqi=255),
                dict(ldgki=100), dict(ldgq=1), dict(ldgk=1), dict(R=3), dict(N=-5)]:
        assert c.get(**bad) == ERR_SHAPE, bad
    for name in ("Q", "K", "pos", "table", "GQ", "GK", "GQin", "GKin", "workspace"):
        assert c.get(**{name: None}) == ERR_NULL, name
    for name in ("Q", "GQ", "GKin", "Gwq", "Gwk", "workspace", "wq"):
        assert c.get(**{name: c.args[name] + 1}) == ERR_ALIGN, name
    for bad in [dict(GQin=A), dict(GQin=F), dict(Gwq=K), dict(workspace=J), dict(workspace=H), dict(GKin=H + 256),
                dict(Gwk=E)]:
        assert c.get(**bad) == ERR_ALIAS, bad


def test_kv_append(lib):
    c = Call(lib.ssn_kv_append, dtype=1, N=10, B=3, Hq=4, Hk=2, D=64, R=64, P=100, style=0, eps=1e-6, Q=A, ldq=512,
             K=A + 512, ldk=512, V=A + 768, ldv=512, wq=B, wk=C, table=D, Kc=E, Vc=F, npages=50, page_size=16,
             pages=G, width=7, starts=H, lens=J, Qout=K, ldqo=256, stream=None)
    assert c.get(dtype=3) == ERR_DTYPE
    assert c.get(N=0, K=None, pages=None) == OK and c.get(B=0, K=None, starts=None) == OK
    for bad in [dict(N=-1), dict(B=-1), dict(B=1 << 20), dict(Hk=0), dict(npages=0), dict(page_size=0), dict(width=0),
                dict(width=1 << 28), dict(npages=1 << 28), dict(page_size=1 << 30), dict(ldv=127), dict(R=65),
                dict(eps=-1.0), dict(N=1 << 31)]:
        assert c.get(**bad) == ERR_SHAPE, bad
    for name in ("Q", "K", "V", "table", "Kc", "Vc", "pages", "starts", "lens", "Qout"):
        assert c.get(**{name: None}) == ERR_NULL, name
    for name in ("Q", "K", "V", "Kc", "Vc", "Qout", "pages", "starts", "lens", "table"):
        assert c.get(**{name: c.args[name] + 1}) == ERR_ALIGN, name
    size = 50 * 16 * 2 * 64 * 2
    for bad in [dict(Vc=E + size - 2), dict(Kc=A), dict(Qout=E), dict(Qout=A), dict(Kc=G), dict(Vc=J), dict(Kc=D)]:
        assert c.get(**bad) == ERR_ALIAS, bad


def test_paged_attention(lib):
    c = Call(lib.ssn_paged_attention, dtype=1, N=10, B=3, Hq=4, Hk=2, D=64, max_q=4, max_len=100, scale=0.125, Q=A,
             ldq=512, Kc=B, Vc=C, npages=50, page_size=16, pages=D, width=7, starts=E, lens=F, O=G, ldo=256, lse=H,
             workspace=J, bytes=1 << 20, stream=None)
    assert c.get(dtype=2) == ERR_DTYPE
    assert c.get(N=0, Q=None, O=None) == OK and c.get(B=0, Q=None) == OK
    for bad in [dict(N=-1), dict(B=-1), dict(Hq=3), dict(Hq=0), dict(Hk=0), dict(D=0), dict(max_q=-1),
                dict(max_len=-1), dict(max_len=1 << 31), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(ldq=255), dict(ldo=100), dict(npages=0), dict(page_size=0), dict(width=0), dict(width=1 << 30),
                dict(npages=1 << 27), dict(N=1 << 30, Hq=4), dict(bytes=(1 << 64) - 1), dict(bytes=1 << 63)]:
        assert c.get(**bad) == ERR_SHAPE, bad
    assert c.get(D=1025, ldq=1 << 13, ldo=1 << 13) == ERR_UNSUPPORTED
    for name in ("Q", "Kc", "Vc", "pages", "starts", "lens", "O", "workspace"):
        assert c.get(**{name: None}) == ERR_NULL, name
    for name in ("Q", "Kc", "Vc", "pages", "starts", "lens", "O", "lse"):
        assert c.get(**{name: c.args[name] + 1}) == ERR_ALIGN, name
    assert c.get(workspace=J + 8) == ERR_ALIGN
    for bad in [dict(O=A), dict(O=A + 256, ldo=512), dict(O=B), dict(lse=G), dict(workspace=H - (1 << 19)),
                dict(O=F), dict(workspace=C)]:
        assert c.get(**bad) == ERR_ALIAS, bad
    w = lib.ssn_paged_attention_workspace_bytes
    assert w(1, 0, 3, 4, 2, 64, 4, 100) == 0 and w(9, 10, 3, 4, 2, 64, 4, 100) == 0
    assert w(1, 10, 3, 3, 2, 64, 4, 100) == 0 and w(1, 10, 3, 4, 2, 4096, 4, 100) == 0
    assert w(1, 10, -3, 4, 2, 64, 4, 100) == 0 and w(1, 10, 3, 4, 2, 64, -4, 100) == 0


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and the HIP headers")
def test_validation_is_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "attn_asan")
    src, here = os.path.join(ROOT, "paper_2607_13332_amd", "csrc"), os.path.join(ROOT, "tests", "asan")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I" + os.path.join(ROOT, "include"), "-I" + src, "-x", "c++", os.path.join(src, "attn_api.hip"),
           "-x", "none", os.path.join(here, "attn_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "attention validation ok" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
