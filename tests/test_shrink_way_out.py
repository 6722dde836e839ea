"""CPU: the shrinking product of the adapters leaves its sums where its stages were.  When a wait has run out copies may still be on their way
there: the marks that say so (NaN) are written once those have landed.  The source is read: it cannot be provoked on purpose."""
import pathlib
import re

TEXT = (pathlib.Path(__file__).resolve().parent.parent / "paper_2604_06916_b200" / "csrc" / "lora_apply.cu").read_text()


def test_marks_are_written_behind_the_copies():
    start = TEXT.index("w * kShrinkWindow < t1 - t0")
    part = TEXT[start:TEXT.index("cluster_sync()", start)]
    pause = re.search(r"if \(!ok\) __nanosleep\((\d+)\);", part)
    assert pause and int(pause.group(1)) >= 1_000_000
    assert pause.start() < part.index("float *mine") < part.index("make_float4(nan")
