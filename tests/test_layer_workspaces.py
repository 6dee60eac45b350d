"""Workspaces of the entry points around the experts' products: their sizes, and what is refused of them -- missing, one word short, unaligned, on top of another buffer.  Without a GPU: nothing
here is launched.  Once more in a child process under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import subprocess
import sys

import pytest

import test_host_sanitizers as S
from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import build as BUILD

P = [0x400000000 * (i + 1) for i in range(12)]                         # addresses far from each other; never touched


def norm(T, H, dw=P[5], ws=P[6], n=None, off=0, **kw):
    d = B.RmsNormDesc(T, H, B.AXE_BF16, B.AXE_BF16, **kw)
    words = B.lib().axe_rmsnorm_workspace(d.ref)
    return words, B.lib().axe_rmsnorm_backward(d.ref, P[0], P[1], P[2], P[3], P[4], dw, ws, words + off if n is None else n, None)


# workgroups of rows in turns: 8 rows of up to 512 columns, 1024 / threads of wider ones, at most 512 workgroups; none for one workgroup
@pytest.mark.parametrize("T,H,words", [(1, 2048, 0), (8, 2048, 0), (9, 2048, 3 * 2048), (64, 2048, 16 * 2048), (4096, 2048, 512 * 2048), (2, 20000, 0), (3, 20000, 3 * 20000), (16, 7, 0), (17, 7, 21),
                                       (100000, 64, 512 * 64), (100, 1000, 13 * 1000), (5, 8192, 3 * 8192)])
def test_norm_workspace(T, H, words):
    assert norm(T, H)[0] == words
    if words == 0:
        return
    for bad in (dict(ws=None), dict(off=-1), dict(n=0), dict(n=-1), dict(ws=P[6] + 2), dict(ws=P[0]), dict(ws=P[1] + 64), dict(ws=P[2]), dict(ws=P[3]), dict(ws=P[4]), dict(ws=P[5]),
                dict(ws=P[5] + 4 * (H - 1)), dict(ws=P[4] - 4 * words + 4)):
        assert norm(T, H, **bad)[1] == B.AXE_EINVAL, bad


def route(T, E, k, ws=P[6], n=None, off=0, rows=P[3], ro=P[4]):
    d = B.RouteDesc(T, E, k)
    words = B.lib().axe_route_workspace(d.ref)
    return words, B.lib().axe_route(d.ref, P[0], P[1], P[2], rows, ro, ws, words + off if n is None else n, None)


# 16-bit counts of the experts, rounded up to a power of two of at least 8, for blocks of 8, 16, 32 and more tokens; none for one workgroup
@pytest.mark.parametrize("T,E,k,words", [(1, 128, 8, 0), (64, 128, 8, 0), (65, 128, 8, 9 * 64), (48, 256, 8, 0), (49, 256, 8, 7 * 128), (32, 512, 8, 0), (33, 512, 8, 5 * 256), (2048, 60, 4, 256 * 32),
                                         (2049, 60, 4, 129 * 32), (5000, 32, 4, 157 * 16), (8193, 8, 2, 171 * 4), (33333, 1000, 8, 232 * 512), (1 << 24, 9, 1, 257 * 8)])
def test_route_workspace(T, E, k, words):
    assert route(T, E, k)[0] == words
    if words == 0:
        return
    for bad in (dict(ws=None), dict(off=-1), dict(n=0), dict(n=-1), dict(ws=P[6] + 2), dict(ws=P[0]), dict(ws=P[1]), dict(ws=P[2]), dict(ws=P[3]), dict(ws=P[4]), dict(ws=P[1] - 4 * words + 4)):
        assert route(T, E, k, **bad)[1] == B.AXE_EINVAL, bad


def test_under_address_and_undefined_behaviour_sanitizers():
    if os.environ.get("AXE_TEST_HOST_LIB"):
        return                                             # this is the child run itself
    if not os.path.exists(S.SAN_LIB):
        BUILD.build_hostcheck_sanitized()
    env = dict(os.environ)
    env["LD_PRELOAD"] = ":".join(filter(None, [env.get("LD_PRELOAD", ""), BUILD.sanitizer_runtime()]))
    env["ASAN_OPTIONS"] = "detect_leaks=0:verify_asan_link_order=0:abort_on_error=0"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    env["AXE_TEST_HOST_LIB"] = S.SAN_LIB
    p = subprocess.run([sys.executable, "-m", "pytest", "tests/test_layer_workspaces.py", "-x", "-q", "-m", "not gpu", "-p", "no:cacheprovider"],
                       cwd=S.ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=900)
    assert "AddressSanitizer" not in p.stdout and "runtime error:" not in p.stdout, p.stdout[-4000:]
    assert p.returncode == 0 and " passed" in p.stdout, p.stdout[-4000:]
