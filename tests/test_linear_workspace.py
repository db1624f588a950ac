"""The linear layers' workspace size without an object, on the CPU; on the GPU the example's
layers, which share one."""
import importlib.util
import os

import pytest
import torch

from paper_2602_03839_amd import head

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "block_loop.py")


def test_size_without_an_object():
    size = head.linear_workspace_bytes
    for tokens, rows, cols in ((77, 1003, 203), (4096, 18944, 3584), (1, 1, 1)):
        assert size(tokens, rows, cols) == head.lib().pulse_linear_workspace_bytes(tokens, rows, cols) > 0
        # every part of two BF16 values of d, and of the tokens, is in it
        assert size(tokens, rows, cols) >= tokens * (rows * 4 + cols * 2)
    top = head.LINEAR_MAX_WIDTH
    assert size(0, 64, 64) == size(5, 0, 64) == size(5, 64, top + 1) == size(-1, 64, 64) == size(1 << 33, 64, 64) == 0
    assert size(top, top, top) > 0


@pytest.mark.gpu
def test_the_examples_layers_share_one():
    spec = importlib.util.spec_from_file_location("block_loop", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    policy = m.Policy(m.masters(300, 136, 264, g), 100)
    layers = (policy.gate, policy.up, policy.down, policy.head)
    assert len({layer.ws.data_ptr() for layer in layers}) == 1
    for layer in layers:
        need = head.linear_workspace_bytes(100, layer.rows, layer.cols)
        assert layer.workspace_bytes == need <= layer.ws.numel()
