"""A call's stream has to belong to the device of its tensors: a kernel on another one would not reach them."""
import os
from types import SimpleNamespace

import pytest
import torch

from paper_2602_16052_amd import binding as mb


def stream_of(index):
    return SimpleNamespace(device=torch.device("cuda", index), device_index=index, cuda_stream=0)


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(mb.LIB_PATH):
        from paper_2602_16052_amd import build
        build.build_library()
    return mb.load_library()


def test_a_stream_of_another_device_is_refused():
    with pytest.raises(ValueError, match="stream must belong to cuda:0, got one of cuda:1"):
        mb._Call("moespec_block_norm", torch.device("cuda", 0), (), (), stream_of(1))
    mb._Call("moespec_block_norm", torch.device("cuda", 1), (), (), stream_of(1))
    mb._Call("moespec_block_norm", torch.device("cuda", 1), (), (), None)
