"""Buffer sizes whose bytes 64 bits do not hold, at the entry points around the experts' products: refused, and not computed with; sizes of buffers that are not given are not looked at.
Without a GPU, and once more under the sanitizers."""
import os
import subprocess
import sys

import pytest

import test_host_sanitizers as S
from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import build as BUILD

P = [0x400000000 * (i + 1) for i in range(12)]                         # addresses far from each other; never touched
HUGE = [1 << 59, 1 << 61, 1 << 62, (1 << 63) - 1]


@pytest.mark.parametrize("elems", HUGE)
def test_norm(elems):
    L = B.lib()
    for field in ("x_elems", "residual_elems", "sum_elems", "y_elems"):
        d = B.RmsNormDesc(4, 64, B.AXE_F32, B.AXE_F32)
        setattr(d.c, field, elems)
        assert L.axe_rmsnorm(d.ref, P[0], P[1], P[2], P[3], P[4], None, None) == B.AXE_EINVAL, field
        assert L.axe_rmsnorm_backward(d.ref, P[0], P[1], P[2], P[3], P[4], None, None, 0, None) == B.AXE_EINVAL, field
        assert b"elements" in L.axe_last_error()


@pytest.mark.parametrize("elems", HUGE)
def test_sizes_of_buffers_that_are_not_given_do_not_matter(elems):
    """(What is refused here is the overlap of y with x.)"""
    d = B.RmsNormDesc(4, 64, B.AXE_F32, B.AXE_F32)
    d.c.residual_elems = d.c.sum_elems = elems
    assert B.lib().axe_rmsnorm(d.ref, P[0], None, P[2], None, P[0] + 4, None, None) == B.AXE_EINVAL
    assert b"overlaps" in B.lib().axe_last_error()
    d = B.RmsNormDesc(4, 64, B.AXE_F32, B.AXE_F32)
    d.c.residual_elems = elems
    assert B.lib().axe_rmsnorm_backward(d.ref, P[0], P[1], P[2], None, P[0] + 4, None, None, 0, None) == B.AXE_EINVAL
    assert b"overlaps" in B.lib().axe_last_error()


@pytest.mark.parametrize("elems", HUGE)
def test_routing_and_rows(elems):
    L = B.lib()
    d = B.RouteDesc(4, 32, 4)
    d.c.logits_elems = elems
    assert L.axe_route(d.ref, P[0], P[1], P[2], None, None, None, 0, None) == B.AXE_EINVAL
    assert L.axe_route_backward(d.ref, P[0], P[1], P[2], P[3], None) == B.AXE_EINVAL
    for field in ("tokens_elems", "rows_elems"):
        d = B.RowsDesc(4, 2, 8, 64, B.AXE_F32, B.AXE_F32)
        setattr(d.c, field, elems)
        assert L.axe_rows_dispatch(d.ref, P[0], None, P[1], P[2], None, None) == B.AXE_EINVAL, field
        assert L.axe_rows_combine(d.ref, P[0], P[1], P[2], P[3], P[4], None) == B.AXE_EINVAL, field
        assert L.axe_rows_combine_backward(d.ref, P[0], P[1], P[2], P[3], P[4], P[5], None) == B.AXE_EINVAL, field
        assert b"elements" in L.axe_last_error()


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
    p = subprocess.run([sys.executable, "-m", "pytest", "tests/test_layer_huge_sizes.py", "-x", "-q", "-m", "not gpu", "-p", "no:cacheprovider"],
                       cwd=S.ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=900)
    assert "AddressSanitizer" not in p.stdout and "runtime error:" not in p.stdout, p.stdout[-4000:]
    assert p.returncode == 0 and " passed" in p.stdout, p.stdout[-4000:]
