"""What the attention for drafted tokens takes from its registers, in the built code: two work-groups per compute unit (at most 256 of a
lane's 512), no values kept in memory (a share's bookkeeping that went there has come back wrong), and no loops over lanes around
loads, whose addresses are the same for a whole wave."""
import os
import re
import subprocess

import pytest

from paper_2201_05596_amd import build as B

LLVM = "/opt/rocm/llvm/bin"


@pytest.fixture(scope="module", params=["bf16", "fp8", "fp4"])
def built(request, tmp_path_factory):
    obj, tmp = os.path.join(B.HERE, "_build", f"tree_attn_{request.param}.o"), tmp_path_factory.mktemp("tree")
    fat, co = str(tmp / "f.fat"), str(tmp / "f.co")
    if not os.path.exists(obj) or not os.path.exists(LLVM + "/llvm-readelf"):
        pytest.skip("needs the built object file and llvm-readelf")
    subprocess.run([LLVM + "/llvm-objcopy", "--dump-section", ".hip_fatbin=" + fat, obj, os.devnull], check=True, capture_output=True)
    subprocess.run([LLVM + "/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                    "--input=" + fat, "--output=" + co], check=True, capture_output=True)
    run = lambda *a: subprocess.run(a, check=True, capture_output=True, text=True).stdout  # noqa: E731
    return run(LLVM + "/llvm-readelf", "--notes", co), run(LLVM + "/llvm-objdump", "-d", co)


def test_registers_and_scratch(built):
    found = re.findall(r"\.name: +\S*?tree_attn_kernelI((?:Li\d+E)+)E\S*.*?\.private_segment_fixed_size: +(\d+).*?\.vgpr_count: +(\d+)", built[0], re.S)
    assert len(found) == 2 * 4
    for args, scratch, registers in found:
        assert int(scratch) == 0 and int(registers) <= 256, args


def test_no_loops_over_lanes_around_loads(built):
    for kernel in built[1].split("<_ZN3moe16tree_attn_kernel")[1:]:
        code = [line.split("//")[0] for line in kernel.splitlines()]
        # such a loop ends by taking the lanes that are served out of exec, right behind the load
        assert not any("s_xor_b64 exec" in b and "buffer_load" in a for a, b in zip(code, code[1:])), kernel.splitlines()[0]
