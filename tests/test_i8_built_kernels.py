"""What the built library holds for 8-bit experts: no kernel that no call reaches, none that keeps values in scratch memory."""
import os
import re
import subprocess

import pytest

from paper_2201_05596_amd import build as B
from tests.test_tree_occupancy import LLVM, code_objects


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """mangled name -> (registers, bytes of scratch memory) of every kernel of the library"""
    if not os.path.exists(B.LIB) or not os.path.exists(LLVM + "/llvm-readelf"):
        pytest.skip("needs the built library and llvm-readelf")
    path, found = str(tmp_path_factory.mktemp("code") / "co"), {}
    for code in code_objects(B.LIB):
        with open(path, "wb") as f:
            f.write(code)
        notes = subprocess.run([LLVM + "/llvm-readelf", "--notes", path], check=True, capture_output=True, text=True).stdout
        for name, scratch, registers in re.findall(r"\.name: +(_Z\S+).*?\.private_segment_fixed_size: +(\d+).*?\.vgpr_count: +(\d+)", notes, re.S):
            found[name] = (int(registers), int(scratch))
    return found


def test_gate_finds_rows_maxima_for_few_tokens_only(kernels):
    """gate_decode_kernel<MA, RK, NV, PLAIN, MAXES>: layers that let it find the tokens' largest magnitudes have up to 128 tokens, tiles of 16 (MA = 1)."""
    found = [tuple(map(int, re.findall(r"L[ib](\d+)E", n))) for n in kernels if "gate_decode_kernel" in n]
    assert len(set(found)) == len(found) and {m for m in found if not m[4]} == {(ma, rk, nv, plain, 0) for ma in (1, 2) for rk in (1, 2) for nv in (1, 2, 4, 8) for plain in (0, 1)}
    assert {m for m in found if m[4]} == {(1, rk, nv, plain, 1) for rk in (1, 2) for nv in (1, 2, 4, 8) for plain in (0, 1)}


@pytest.mark.parametrize("name", ["i8_rows_kernel", "i8_weights_kernel", "i8_few_kernel", "i8_token_first_kernel", "i8_token_second_kernel",
                                  "i8_token_gather_kernel", "i8_tile_kernel"])
def test_nothing_in_scratch_memory(kernels, name):
    """Rows and weights are held in registers between their largest magnitude and their codes; and the build refuses a source that does otherwise."""
    found = {n: v for n, v in kernels.items() if name in n}
    assert found and not {n: v for n, v in found.items() if v[1]}
    assert {f"i8_{s}.hip" for s in ("quant", "few", "token", "tile")} <= set(B.NO_SCRATCH)
