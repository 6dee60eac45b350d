"""What is refused of a call on a paged cache does not depend on the thread's calls before it, without a GPU: the analysis of a descriptor's layouts is kept from one call to the next, and two
descriptors that differ in anything it depends on share none."""
import pytest

from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import workloads as W
from test_cache_refusals import P, desc, host

# (pages, tokens of a page, heads, columns) of a cache of 5 pages of 16 tokens, 2 heads of 64 columns: multiples of 8 elements (16 bytes in 16 bits), not of 16 (in e4m3)
OFF = [((2176, 136, 64, 1), 0), ((2304, 144, 72, 1), 0), ((2056, 128, 64, 1), 0), ((2048, 128, 64, 1), 8)]


def layout(strides, offset):
    return B.Layout(W.spec([(n, s, "m") for n, s in zip((5, 16, 2, 64), strides)], O={"m": offset}), ["m"])


def call(entry, L, cache, dt=B.AXE_BF16):
    d = desc(k_cache=L, v_cache=L, k_cache_elems=1 << 16, v_cache_elems=1 << 16, cache=cache, dt=dt)
    s = (P[10], P[11]) if cache == B.AXE_FP8_E4M3 else (None, None)
    if entry == "append":
        return host().axe_cache_append(d.ref, P[0], P[1], P[2], P[3], P[4], P[5], P[6], P[7], P[8], P[9], *s, None)
    return host().axe_cache_attention(d.ref, P[0], P[8], P[9], *s, P[4], P[5], P[6], P[7], P[12], max(0, host().axe_cache_attention_workspace(d.ref)), None)


@pytest.mark.parametrize("entry", ["append", "attention"])
@pytest.mark.parametrize("strides, offset", OFF)
def test_strides_of_an_e4m3_cache_are_refused_after_a_call_in_16_bits_with_the_same_layouts(entry, strides, offset):
    L = layout(strides, offset)
    assert call(entry, L, B.AXE_FP8_E4M3) == B.AXE_EUNSUPPORTED
    for dt in (B.AXE_BF16, B.AXE_F16):
        assert call(entry, L, dt, dt) == B.AXE_EHIP                    # (not refused: the stand-in of the launch is what fails)
        assert call(entry, L, B.AXE_FP8_E4M3, dt) == B.AXE_EUNSUPPORTED, (entry, strides, offset)
        assert call(entry, L, dt, dt) == B.AXE_EHIP


@pytest.mark.parametrize("entry", ["append", "attention"])
def test_a_layout_that_both_types_take_is_taken_in_any_order(entry):
    L = layout((2048, 128, 64, 1), 0)
    for cache in (B.AXE_FP8_E4M3, B.AXE_BF16, B.AXE_FP8_E4M3, B.AXE_BF16):
        assert call(entry, L, cache) == B.AXE_EHIP
