"""What the attention for drafted tokens rests on in the built library: as many work-groups per compute unit as there are shares for
one (a lane has 512 registers for the waves of its SIMD; a unit has 160 KB of LDS), nothing in scratch memory, and what scalar registers
do not hold in lanes of a register of its own."""
import os
import re
import subprocess

import pytest

from paper_2201_05596_amd import build as B

LLVM = "/opt/rocm/llvm/bin"
BITS = [16, 8, 4]


def code_objects(path):
    """The library's code objects for the GPU: each source's bundle is a table of (offset, size, target) behind its magic."""
    data = open(path, "rb").read()
    word = lambda at: int.from_bytes(data[at:at + 8], "little")  # noqa: E731
    for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data):
        at = m.end() + 8
        for _ in range(word(m.end())):
            offset, size, name = word(at), word(at + 8), word(at + 16)
            if b"gfx950" in data[at + 24:at + 24 + name]:
                yield data[m.start() + offset:m.start() + offset + size]
            at += 24 + name


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{(kind, head_dim, tiles of 16 rows, waves with rows of their own): (registers, bytes of scratch, code)}"""
    path, found = str(tmp_path_factory.mktemp("code") / "co"), {}
    run = lambda *a: subprocess.run(a, check=True, capture_output=True, text=True).stdout  # noqa: E731
    for code in code_objects(B.LIB):
        if b"tree_attn_kernel" not in code:
            continue
        with open(path, "wb") as f:
            f.write(code)
        notes = run(LLVM + "/llvm-readelf", "--notes", path)
        text = {m.group(1): m.group(2) for m in re.finditer(r"<(_ZN3moe16tree_attn_kernel\S*)>:\n(.*?)(?=\n\n|\Z)", run(LLVM + "/llvm-objdump", "-d", path), re.S)}
        for name, args, scratch, registers in re.findall(
                r"\.name: +(\S*?tree_attn_kernelI((?:Li\d+E)+)E\S*).*?\.private_segment_fixed_size: +(\d+).*?\.vgpr_count: +(\d+)", notes, re.S):
            found[tuple(map(int, re.findall(r"\d+", args)))] = (int(registers), int(scratch), text[name])
    assert len(found) == 3 * 2 * 4
    return found


def test_work_groups_per_unit(kernels):
    """256 registers for two, 168 for three."""
    for (kind, dh, mt, wr), (registers, _, _) in kernels.items():
        three = wr == 1 and 2 * 32 * dh * BITS[kind] // 8 <= 4096
        assert registers <= (168 if three else 256), (kind, dh, mt, wr)
        # LDS that a launch asks for: the rounds' tiles, or the rows that waves join
        tiles = 4 * (dh // 32 * 2 + dh // 16) * 1024 if wr > 1 else 0
        merge = 4 * 16 * mt * (dh + 4 + 2) * 4 if wr < 4 else 0
        assert (3 if three else 2) * max(tiles, merge) <= 160 * 1024, (kind, dh, mt, wr)


def test_nothing_in_scratch_memory(kernels):
    assert [k for k, (_, scratch, text) in kernels.items() if scratch or "scratch_" in text] == []


def test_lanes_that_hold_scalars_are_written_by_nothing_else(kernels):
    vector = re.compile(r"\bv(?:\[(\d+):(\d+)\]|(\d+)\b)")
    numbers = lambda text: {n for a, b, c in vector.findall(text) for n in range(int(a or c), int(b or c) + 1)}  # noqa: E731
    for key, (_, _, text) in kernels.items():
        code = [line.split("//")[0].strip() for line in text.splitlines()]
        held = set().union(*(numbers(line.split(",")[0]) for line in code if line.startswith("v_writelane")))
        assert held, key
        assert not [line for line in code if not line.startswith(("v_writelane", "v_readlane")) and numbers(line) & held], key


def test_a_build_with_scratch_memory_is_refused():
    remark = lambda name, size: (f"k.h:1:1: remark: Function Name: {name} [-Rpass-analysis=kernel-resource-usage]\n"  # noqa: E731
                                 f"k.h:1:1: remark:     ScratchSize [bytes/lane]: {size} [-Rpass-analysis=kernel-resource-usage]\n")
    assert B.kernels_in_scratch(remark("a", 0) + remark("b", 16) + remark("c", 0)) == ["b"]
    assert B.kernels_in_scratch(remark("a", 0)) == []
    with pytest.raises(RuntimeError):
        B.kernels_in_scratch("")
    assert set(B.NO_SCRATCH) <= set(B.SOURCES)
