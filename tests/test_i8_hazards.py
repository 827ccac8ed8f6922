"""The distances of test_wide_hazards.py in the built kernels on codes.  The compiler leaves behind a 16 x 16 x 64 matrix instruction on
8-bit integers as many wait states as behind a 16 x 16 x 32 one in bf16, 8 passes as well."""
import os
import re
import subprocess

import pytest

from paper_2201_05596_amd import build as B
from tests import test_wide_hazards as H


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """name -> code of the 256-row tiles' and the 128-row tiles' kernels"""
    found = {}
    for name, kernel in (("i8_wide", "wide_kernel"), ("i8_tile", "i8_tile_kernel")):
        obj = os.path.join(B.HERE, "_build", name + ".o")
        if not os.path.exists(obj) or not os.path.exists(H.LLVM + "/llvm-objdump"):
            pytest.skip("needs the built object files and llvm-objdump")
        found[name] = code_of(obj, kernel, str(tmp_path_factory.mktemp(name)))
    return found


def code_of(obj, kernel, folder):
    fat, out = folder + "/a.fat", folder + "/a.co"
    subprocess.run([H.LLVM + "/llvm-objcopy", "--dump-section", ".hip_fatbin=" + fat, obj, os.devnull], check=True, capture_output=True)
    subprocess.run([H.LLVM + "/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                    "--input=" + fat, "--output=" + out], check=True, capture_output=True)
    found, current = {}, None
    for line in subprocess.run([H.LLVM + "/llvm-objdump", "-d", out], check=True, capture_output=True, text=True).stdout.splitlines():
        m = re.match(r"[0-9a-f]+ <(\S+)>:", line)
        if m:
            current = found.setdefault(m.group(1), [])
        elif current is not None and "//" in line:
            body, _, tail = line.partition("//")
            current.append((int(tail.strip().split(":")[0], 16), " ".join(body.split())))
    return {n: c for n, c in found.items() if kernel in n}


def test_built_code_keeps_the_distances(kernels):
    assert kernels["i8_wide"]
    for name, code in kernels["i8_wide"].items():
        assert sum(line.startswith("v_mfma_i32_16x16x64_i8") for _, line in code) >= 224, name
        assert not H.find_hazards(code), name


def test_direct_loads_wait_for_m0(kernels):
    for group in kernels.values():
        assert group
        for name, code in group.items():
            assert sum("_lds_" in line.split()[0] for _, line in code) >= 8
            assert not H.find_m0_hazards(code), name
