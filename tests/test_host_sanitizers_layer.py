"""The argument checks of the entry points around the grouped GEMMs under AddressSanitizer and UndefinedBehaviorSanitizer, as the other files of the host layer
(tests/test_host_sanitizers.py): their refusals once more in a child process."""
import os
import subprocess
import sys

import test_host_sanitizers as S
from paper_2601_19092_amd import build as BUILD


def test_refusals_under_address_and_undefined_behaviour_sanitizers():
    if os.environ.get("AXE_TEST_HOST_LIB"):
        return                                             # this is the child run itself
    if not os.path.exists(S.SAN_LIB):
        BUILD.build_hostcheck_sanitized()
    env = dict(os.environ)
    env["LD_PRELOAD"] = ":".join(filter(None, [env.get("LD_PRELOAD", ""), BUILD.sanitizer_runtime()]))
    env["ASAN_OPTIONS"] = "detect_leaks=0:verify_asan_link_order=0:abort_on_error=0"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    env["AXE_TEST_HOST_LIB"] = S.SAN_LIB
    p = subprocess.run([sys.executable, "-m", "pytest", "tests/test_layer_ops_refusals.py", "-x", "-q", "-m", "not gpu", "-p", "no:cacheprovider"],
                       cwd=S.ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=900)
    assert "AddressSanitizer" not in p.stdout and "runtime error:" not in p.stdout, p.stdout[-4000:]
    assert p.returncode == 0 and " passed" in p.stdout, p.stdout[-4000:]
