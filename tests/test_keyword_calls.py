"""CPU: the entries that run on their first argument's device take it by its name as well as by its place, and refuse what
is not a CUDA tensor in the same way."""
import inspect

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding, build

    build.build()
    binding.lib()
    return binding


ENTRIES = ["nvfp4_matvec", "mxfp4_matvec", "sol_qk_rotary", "sol_qk_rotary_backward", "sol_select_blocks", "sol_attention_blocks"]


@pytest.mark.parametrize("name", ENTRIES)
def test_first_argument_by_name_and_by_place(B, name):
    fn = getattr(B, name)
    names = [p.name for p in inspect.signature(fn).parameters.values()]
    required = [p.name for p in inspect.signature(fn).parameters.values() if p.default is inspect.Parameter.empty]
    host = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16)
    rest = {n: None for n in required[1:]}
    for first in (host, None, 3):                                     # host tensors, nothing, not a tensor
        with pytest.raises(TypeError, match="CUDA"):
            fn(first, **rest)
        with pytest.raises(TypeError, match="CUDA"):
            fn(**{names[0]: first}, **rest)
    with pytest.raises(TypeError, match=names[0]):                    # missing: the message names it
        fn(**rest)
    with pytest.raises(TypeError):                                    # given twice
        fn(host, **{names[0]: host}, **rest)
