"""CPU: what the host side keeps between calls (blocks that fit an SM, clusters that fit the GPU, attributes that are set) it keeps for
each device by itself, and what several threads may write at once is atomic where its value decides how work is shared.  Read from
the source of the training step's operators."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2604_06916_b200" / "csrc"


@pytest.mark.parametrize("name,kept", [("layernorm.cu", 1), ("adamw.cu", 1), ("lora_apply.cu", 2)])
def test_kept_counts(name, kept):
    found = re.findall(r"^ +static (?!constexpr|const )([^;=]*?) (\w+)((?:\[\w+\])*)", (CSRC / name).read_text(), re.M)
    assert len(found) == kept
    for kind, variable, places in found:
        assert places.startswith("[64]"), f"{variable}: one for each device"
        assert kind == "bool" or kind == "std::atomic<int>", f"{variable}: {kind}"
