"""CPU: the training step's entries that run on their first argument's device take it by its name as well as by its place, and refuse
what is not a CUDA tensor in the same way."""
import inspect

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding, build

    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("name", ["sol_layernorm", "sol_layernorm_backward", "sol_lora_apply", "sol_lora_backward"])
def test_first_argument_by_name_and_by_place(B, name):
    fn = getattr(B, name)
    parameters = inspect.signature(fn).parameters.values()
    names, required = [p.name for p in parameters], [p.name for p in parameters if p.default is inspect.Parameter.empty]
    host = torch.zeros((4, 64), dtype=torch.bfloat16)
    rest = {n: None for n in required[1:]}
    for first in (host, None, 3):
        with pytest.raises(TypeError, match="CUDA"):
            fn(first, **rest)
        with pytest.raises(TypeError, match="CUDA"):
            fn(**{names[0]: first}, **rest)
    with pytest.raises(TypeError, match=names[0]):
        fn(**rest)
