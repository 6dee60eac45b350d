"""What the entry points of the paged cache refuse, without a GPU: bad sizes, types, layouts, buffers and workspaces are error codes before anything is launched.  On the host layer with stand-ins
for the kernels (what is not refused ends there, wherever this runs); once more under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import subprocess
import sys

import pytest

import test_host_sanitizers as S
from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import build as BUILD
from paper_2601_19092_amd import workloads as W

def host():
    """The host layer without kernels."""
    if os.environ.get("AXE_TEST_HOST_LIB"):
        return B.lib()
    path = os.path.join(BUILD.HERE, "libaxe_hostcheck.so")
    if path not in _loaded:
        if not os.path.exists(path):
            BUILD.build_hostcheck()
        _loaded[path] = B.load(path)
    return _loaded[path]


_loaded = {}
P = [0x4000000000 * (i + 1) for i in range(14)]                        # addresses far from each other; never touched


def desc(T=6, S=2, Hq=4, Hkv=2, D=64, pages=5, page=16, most=3, dt=B.AXE_BF16, cache=None, set_=None, **kw):
    d = B.CacheDesc(T, S, Hq, Hkv, D, pages, page, most, dt, cache, **kw)
    for f, v in (set_ or {}).items():
        setattr(d.c, f, v)
    return d


def append_rc(q=P[0], k=P[1], v=P[2], rot=P[3], rows=P[4], lens=P[5], table=P[6], out=P[7], kc=P[8], vc=P[9], ks=None, vs=None, **kw):
    d = desc(**kw)
    return host().axe_cache_append(d.ref, q, k, v, rot, rows, lens, table, out, kc, vc, ks, vs, None)


def attention_rc(q=P[0], kc=P[8], vc=P[9], ks=None, vs=None, rows=P[4], lens=P[5], table=P[6], out=P[7], ws=P[12], n=None, **kw):
    d = desc(**kw)
    words = host().axe_cache_attention_workspace(d.ref)
    return host().axe_cache_attention(d.ref, q, kc, vc, ks, vs, rows, lens, table, out, ws, max(words, 0) if n is None else n, None)


BOTH = [append_rc, attention_rc]


@pytest.mark.parametrize("rc", BOTH)
def test_sizes_and_types(rc):
    for field in ("T", "S", "pages", "max_pages"):
        assert rc(set_={field: -1}) == B.AXE_EINVAL, field
    for field in ("q_heads", "kv_heads", "head_dim", "page_tokens"):
        assert rc(set_={field: 0}) == B.AXE_EINVAL, field
        assert rc(set_={field: -8}) == B.AXE_EINVAL, field
    assert rc(set_={"q_heads": 5}) == B.AXE_EINVAL
    assert rc(dt=9) == B.AXE_EINVAL and rc(cache=9) == B.AXE_EINVAL and rc(dt=B.AXE_FP8_E4M3) == B.AXE_EINVAL
    assert rc(dt=B.AXE_F32) == B.AXE_EUNSUPPORTED and rc(dt=B.AXE_BF16, cache=B.AXE_F16) == B.AXE_EUNSUPPORTED and rc(dt=B.AXE_F16, cache=B.AXE_F32) == B.AXE_EUNSUPPORTED
    assert rc(D=60) == B.AXE_EUNSUPPORTED and rc(D=264) == B.AXE_EUNSUPPORTED and rc(D=72, cache=B.AXE_FP8_E4M3) == B.AXE_EUNSUPPORTED
    assert rc(Hq=129, Hkv=1) == B.AXE_EUNSUPPORTED
    assert rc(set_={"max_pages": 1 << 28, "page_tokens": 1 << 10}) == B.AXE_EUNSUPPORTED and rc(set_={"S": 1 << 20}) == B.AXE_EUNSUPPORTED
    assert rc(set_={"T": (1 << 30) + 1}) == B.AXE_EUNSUPPORTED and rc(set_={"pages": (1 << 30) + 1}) == B.AXE_EUNSUPPORTED
    # nothing to do: nothing looked at
    assert rc(T=0, q=None, kc=None, vc=None, rows=None, lens=None, table=None, out=None) == B.AXE_OK
    assert rc(S=0, q=None, kc=None, vc=None, rows=None, lens=None, table=None, out=None) == B.AXE_OK


@pytest.mark.parametrize("rc", BOTH)
def test_layouts(rc):
    assert call(rc) == B.AXE_EHIP
    for which, n in (("q", 4), ("out", 4)):
        for bad, want in ((W.spec([(6, 64 * n, "m"), (n, 64, "m"), (64, 2, "m")]), B.AXE_EUNSUPPORTED), (W.spec([(6, 64 * n, "m"), (n * 64, 1, "m")], O={"m": 1}), B.AXE_ERANGE),
                          (W.spec([(6, 64 * n, "m"), (n * 32, 1, "m")]), B.AXE_ESHAPE), (W.spec([(6, 64 * n, "m"), (n * 64, 1, "m")], R=[(2, 4096, "m")]), B.AXE_EUNSUPPORTED),
                          (W.spec([(6, 64 * n, "m"), (2, 64 * n // 2, "m"), (2, -64, "m"), (64, 1, "m")], O={"m": 64}), B.AXE_EUNSUPPORTED)):
            small = {B.AXE_ERANGE: 6 * 64 * n}.get(want, 1 << 20)
            d = {which: B.Layout(bad, ["m"]), which + "_elems": small}
            assert call(rc, **d) == want, (which, bad)
    # out: two heads in one place
    assert call(rc, out=B.Layout(W.spec([(6, 256, "m"), (4, 32, "m"), (64, 1, "m")]), ["m"]), out_elems=1 << 20) == B.AXE_EALIAS
    for which in ("k_cache", "v_cache"):
        for bad, want in ((W.spec([(5, 2048, "m"), (16, 128, "m"), (2, 64, "m"), (64, 1, "m")], O={"m": 4}), B.AXE_EUNSUPPORTED),
                          (W.spec([(5, 2052, "m"), (16, 128, "m"), (2, 64, "m"), (64, 1, "m")]), B.AXE_EUNSUPPORTED),
                          (W.spec([(5, 4096, "m"), (16, 132, "m"), (2, 64, "m"), (64, 1, "m")]), B.AXE_EUNSUPPORTED),
                          (W.spec([(5, 2048, "m"), (16, 64, "m"), (2, 64, "m"), (64, 1, "m")]), B.AXE_EALIAS),
                          (W.spec([(5, 2048, "m"), (16, 128, "m"), (128, 1, "m")], O={"m": 8}), B.AXE_ERANGE)):
            assert call(rc, **{which: B.Layout(bad, ["m"]), which + "_elems": 5 * 2048 if want == B.AXE_ERANGE else 1 << 20}) == want, bad
    for which in ("q", "out", "k_cache", "v_cache"):
        assert call(rc, set_={which + "_elems": 1 << 59}) == B.AXE_EINVAL and b"elements" in host().axe_last_error()
        assert call(rc, set_={which + "_elems": (1 << 63) - 1}) == B.AXE_EINVAL


def call(rc, **kw):
    """The call with layouts that have the names of its buffers."""
    d = desc(**kw)
    if rc is append_rc:
        return host().axe_cache_append(d.ref, P[0], P[1], P[2], P[3], P[4], P[5], P[6], P[7], P[8], P[9], None, None, None)
    return host().axe_cache_attention(d.ref, P[0], P[8], P[9], None, None, P[4], P[5], P[6], P[7], P[12], max(0, host().axe_cache_attention_workspace(d.ref)), None)


def test_append_buffers():
    for name in ("k", "v", "rows", "lens", "table", "kc", "vc"):
        assert append_rc(**{name: None}) == B.AXE_EINVAL, name
    assert append_rc(rot=None, rotary_dim=64) == B.AXE_EINVAL
    assert append_rc(q=None) == B.AXE_EINVAL and append_rc(out=None) == B.AXE_EINVAL
    for name, at in (("q", P[0]), ("k", P[1]), ("out", P[7]), ("rows", P[4]), ("lens", P[5]), ("table", P[6])):
        assert append_rc(**{name: at + 1}) == B.AXE_EINVAL, name
    assert append_rc(kc=P[8] + 8) == B.AXE_EINVAL and append_rc(vc=P[9] + 2) == B.AXE_EINVAL
    assert append_rc(rotary_dim=3) == B.AXE_EINVAL and append_rc(rotary_dim=66) == B.AXE_EINVAL and append_rc(rotary_dim=-2) == B.AXE_EINVAL and append_rc(rotary_style=2) == B.AXE_EINVAL
    assert append_rc(ks=P[10]) == B.AXE_EINVAL and append_rc(cache=B.AXE_FP8_E4M3) == B.AXE_EINVAL and append_rc(cache=B.AXE_FP8_E4M3, ks=P[10]) == B.AXE_EINVAL
    assert append_rc(cache=B.AXE_FP8_E4M3, ks=P[10], vs=P[10] + 4) == B.AXE_EINVAL
    assert append_rc(kc=P[1]) == B.AXE_EINVAL and append_rc(vc=P[8] + 16) == B.AXE_EINVAL and append_rc(vc=P[8]) == B.AXE_EINVAL and append_rc(out=P[1]) == B.AXE_EINVAL
    assert append_rc(out=P[0] + 64) == B.AXE_EINVAL and append_rc(kc=P[6]) == B.AXE_EINVAL and append_rc(out=P[4]) == B.AXE_EINVAL and append_rc(vc=P[7] + 16) == B.AXE_EINVAL


def test_append_queries_in_place_among_keys_and_values():
    """The three in one product's rows, the queries turned where they lie: not refused (the stand-in of the launch is what fails); rows that run into each other are."""
    T, D = 6, 64
    of = lambda at, h, pitch=512: B.Layout(W.spec([(T, pitch, "m"), (h, D, "m"), (D, 1, "m")], O={"m": at}), ["m"])  # noqa: E731

    def rc(**kw):
        d = desc(rotary_dim=64, **kw)
        for f in ("q_elems", "k_elems", "v_elems", "out_elems"):
            setattr(d.c, f, 6 * 512)
        return host().axe_cache_append(d.ref, P[0], P[0], P[0], P[3], P[4], P[5], P[6], P[0], P[8], P[9], None, None, None)

    assert rc(q=of(0, 4), k=of(256, 2), v=of(384, 2), out=of(0, 4)) == B.AXE_EHIP
    assert rc(q=of(0, 4), k=of(192, 2), v=of(384, 2), out=of(0, 4)) == B.AXE_EINVAL
    assert rc(q=of(0, 4), k=of(256, 2), v=of(384, 2), out=of(64, 4)) == B.AXE_EINVAL
    assert rc(q=of(0, 4), k=of(256, 2), v=of(384, 2), out=of(256, 4)) == B.AXE_EINVAL


def test_caches_in_one_buffer():
    """Keys and values of a page side by side, pages apart: not refused; one on top of the other: refused."""
    for off, ok in ((2048, True), (1024, False), (0, False), (4096, False), (4096 * 5, True)):
        L = lambda o: B.Layout(W.spec([(5, 4096, "m"), (16, 128, "m"), (128, 1, "m")], O={"m": o}), ["m"])  # noqa: E731
        d = desc(k_cache=L(0), v_cache=L(off), k_cache_elems=4096 * 12, v_cache_elems=4096 * 12)
        rc = host().axe_cache_append(d.ref, P[0], P[1], P[2], P[3], P[4], P[5], P[6], P[7], P[8], P[8], None, None, None)
        assert rc == B.AXE_EHIP if ok else rc == B.AXE_EINVAL, off


def test_attention_buffers():
    for name in ("q", "kc", "vc", "rows", "lens", "table", "out"):
        assert attention_rc(**{name: None}) == B.AXE_EINVAL, name
    for name, at in (("q", P[0]), ("out", P[7]), ("rows", P[4]), ("lens", P[5]), ("table", P[6])):
        assert attention_rc(**{name: at + 1}) == B.AXE_EINVAL, name
    assert attention_rc(kc=P[8] + 8) == B.AXE_EINVAL and attention_rc(vc=P[9] + 2) == B.AXE_EINVAL
    assert attention_rc(ks=P[10]) == B.AXE_EINVAL and attention_rc(cache=B.AXE_FP8_E4M3) == B.AXE_EINVAL
    for scale in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        assert attention_rc(scale=scale) == B.AXE_EINVAL, scale
    assert attention_rc(window=-1) == B.AXE_EINVAL and attention_rc(window=4, causal=False) == B.AXE_EUNSUPPORTED
    assert attention_rc(out=P[0]) == B.AXE_EINVAL and attention_rc(out=P[8] + 64) == B.AXE_EINVAL and attention_rc(out=P[6]) == B.AXE_EINVAL
    assert host().axe_cache_attention_workspace(desc().ref) == 0 and attention_rc(ws=None) == B.AXE_EHIP   # (few keys: no parts)
    assert host().axe_cache_attention_workspace(desc(most=300).ref) > 0
    for kw in (dict(n=0), dict(ws=None), dict(ws=P[7]), dict(ws=P[12] + 4)):
        assert attention_rc(most=300, **kw) == B.AXE_EINVAL, kw
    assert host().axe_cache_attention_workspace(desc(T=0).ref) == 0 and host().axe_cache_attention_workspace(desc(D=60).ref) == B.AXE_EUNSUPPORTED
    assert host().axe_cache_attention_workspace(None) == B.AXE_EINVAL
    assert host().axe_cache_attention(None, *[None] * 10, 0, None) == B.AXE_EINVAL and host().axe_cache_append(None, *[None] * 13) == B.AXE_EINVAL


def test_a_cache_without_pages_needs_no_buffers():
    for rc in BOTH:
        assert rc(pages=0, kc=None, vc=None) == B.AXE_EHIP


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
    p = subprocess.run([sys.executable, "-m", "pytest", "tests/test_cache_refusals.py", "-x", "-q", "-m", "not gpu", "-p", "no:cacheprovider"],
                       cwd=S.ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=900)
    assert "AddressSanitizer" not in p.stdout and "runtime error:" not in p.stdout, p.stdout[-4000:]
    assert p.returncode == 0 and " passed" in p.stdout, p.stdout[-4000:]


def test_workspaces_follow_from_sizes():
    """Words for the partial results of all workgroups: none where every tile is a workgroup's; the same for the same sizes; enough for the rows of a tile."""
    words = lambda **kw: host().axe_cache_attention_workspace(desc(**kw).ref)  # noqa: E731
    part = lambda rows, cols: 2 * (512 if cols <= 128 else 256) * (4 + 2 * rows + rows * cols)  # noqa: E731
    assert words(T=2, S=2, most=300) == part(16, 64) and words(T=1, S=1, Hq=32, Hkv=4, D=128, most=100) == part(16, 128)
    assert words(T=2, S=2, Hq=32, Hkv=1, most=300) == part(32, 64)     # 32 rows for a token
    assert words(T=80, S=2, most=300) == part(32, 64) and words(T=1600, S=2, most=300) == part(128, 64)      # 4 wide tiles, 50
    assert words(T=100, S=1, Hq=64, Hkv=1, D=256, most=300) == part(128, 256) and words(T=20, S=1, Hq=48, Hkv=48, D=256, most=300) == part(32, 256)
    assert words(T=40, S=1, Hq=48, Hkv=48, D=256, most=300) == part(48, 256)
    assert words(T=1 << 20, S=2, most=300) == 0                        # tiles enough
    assert words(T=5000, S=5000, most=300) == 0                        # more sequences than are cut
    assert words(T=2, S=2, most=48) == 0 and words(T=2, S=2, most=49) > 0   # 768 keys, 784
    assert words(T=32, S=32, most=96) == 0 and words(T=32, S=32, most=97) > 0 and words(T=31, S=31, most=96) > 0
    for kw in (dict(T=2, S=2, most=300), dict(T=600, S=3, Hq=8, Hkv=2, most=200), dict(T=2400, S=3, Hq=8, Hkv=2, most=200)):
        assert words(**kw) == words(**kw, window=100000) and words(**kw) > 0
        assert words(cache=B.AXE_FP8_E4M3, **kw) == words(**kw)
