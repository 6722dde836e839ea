"""CPU: every kernel whose waits are bounded lets its copies in flight land before a CTA leaves that gave a wait up (its shared
memory belongs to the next CTA then).  The source is read: what goes wrong without it cannot be provoked on purpose."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2604_06916_b200" / "csrc"
SOURCES = sorted(p.name for p in CSRC.glob("*.cu") if re.search(r"\bwait_bounded\(", p.read_text()))


def test_kernels_with_bounded_waits_are_found():
    assert {"gemm.cu", "gemm_pair.cu", "gemm_pair_fp4.cu", "attention.cu", "attention_blocks.cu", "matvec.cu"} <= set(SOURCES)


@pytest.mark.parametrize("name", SOURCES)
def test_copies_land_before_a_cta_that_gave_up_leaves(name):
    text = (CSRC / name).read_text()
    out = re.search(r"if \((?:aligned && )?\*abort_flag\) __nanosleep\((\d+)\);", text)
    assert out and int(out.group(1)) >= 1_000_000
    freed = re.search(r"tmem_dealloc(_pair)?\(", text).start()
    barrier = re.search(r"__syncthreads\(\)|cluster_sync\(\)", text[out.end():])
    assert barrier and out.end() + barrier.start() < freed, "the whole CTA waits, and tensor memory is freed after that"
