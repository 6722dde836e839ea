"""CPU: a block that finds nothing to do in a kernel that may start before the one in front of it is done waits for that one before it
leaves.  Else a grid without any work would be done first, and what is launched next, ordered behind it alone, would not find
what the kernels before it write.  The source is read: whether it goes wrong is a matter of timing."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2604_06916_b200" / "csrc"
TEXT = (CSRC / "lora_apply.cu").read_text()
KERNELS = sorted(set(re.findall(r"launch<true>\((\w+)", TEXT)))


def body(name):
    start = re.search(r"__launch_bounds__\([^)]*\)\s*" + name + r"\(", TEXT).end()
    return TEXT[start:TEXT.index("\n}\n", start)]


def test_kernels_are_found():
    assert KERNELS == ["add_slices", "expand_kernel", "outer_kernel"]


@pytest.mark.parametrize("name", KERNELS)
def test_every_way_out_waits(name):
    text = body(name)
    assert "grid_dependency_wait()" in text
    leaves = list(re.finditer(r"\n    if [^\n]*\breturn\b[^\n]*|[^\n]*\breturn;[^\n]*", text))
    for leave in leaves:
        waited = re.search(r"\n    ptx::grid_dependency_wait\(\);", text[:leave.start()])       # not under a condition
        assert waited or "grid_dependency_wait()" in leave.group(), leave.group().strip()
    assert leaves
