"""Registers of the kernels of attention over a paged cache, as hipcc reports them in the built objects (CPU only).  Those that keep everything in registers must not begin to spill unnoticed: tiles of 16 rows at all
sizes, and everything over 16-bit caches but the split kernels of 32 rows of 256 columns."""
import os
import re
import subprocess

import pytest

from paper_2601_19092_amd import build as BLD

LLVM = "/opt/rocm/llvm/bin"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{(type, e4m3, columns, row tiles, split): (registers in memory, bytes of memory)}"""
    out, found = tmp_path_factory.mktemp("isa"), {}
    for source in ("kernels_cache_attention.hip", "kernels_cache_attention_16.hip", "kernels_cache_attention_32.hip"):
        obj = os.path.join(BLD.HERE, "_build", source + ".o")
        if not os.path.exists(obj) or os.path.getmtime(obj) < os.path.getmtime(os.path.join(BLD.CSRC, "cache_attention.h")):
            obj = str(out / (source + ".o"))
            subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *BLD.FLAGS, "-c", os.path.join(BLD.CSRC, source), "-o", obj], stderr=subprocess.DEVNULL)
        fat, code = str(out / (source + ".fat")), str(out / (source + ".co"))
        subprocess.check_call([f"{LLVM}/llvm-objcopy", "--dump-section", f".hip_fatbin={fat}", obj, str(out / "copy.o")])
        subprocess.check_call([f"{LLVM}/clang-offload-bundler", "--type=o", "--unbundle", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={fat}", f"--output={code}"])
        notes = subprocess.check_output([f"{LLVM}/llvm-readelf", "--notes", code], text=True)
        for k in re.split(r"\n\s+- \.agpr_count:", notes)[1:]:
            field = lambda name: int(re.search(rf"\.{name}:\s+(\d+)", k).group(1))  # noqa: E731,B023
            m = re.search(r"cache_attention_kernelILi(\d)ELb(\d)ELi(\d+)ELi(\d)ELb(\d)E", k)
            if m:
                found[tuple(int(x) for x in m.groups())] = field("vgpr_spill_count"), field("private_segment_fixed_size")
    return found


def test_all_kernels_are_there(kernels):
    assert set(kernels) == {(t, fp8, d, rt, split) for t in (1, 4) for fp8 in (0, 1) for d in (64, 128, 256) for rt in (0, 1, 2) for split in (0, 1)}


def test_kernels_without_registers_in_memory(kernels):
    for (t, fp8, d, rt, split), spilt in kernels.items():
        if rt == 1 or d == 64 or (not fp8 and not (rt == 2 and d == 256 and split)):
            assert spilt == (0, 0), (t, fp8, d, rt, split)
