"""The sizes of work buffers that the binding names, against those that the library asks for, without a GPU."""
import ctypes as C

import pytest
import torch

import paper_2601_02311_b200.ps as ps
from test_layer_refusals import LinearDesc, NormDesc

CODES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("tokens, inputs, outputs", [(1, 8, 8), (600, 40, 70), (5003, 1416, 2503)])
def test_linear_buffer_is_large_enough(activation, tokens, inputs, outputs):
    def needed(dtype, wide):
        return ps._lib.ps_linear_backward_bytes(C.byref(LinearDesc(tokens, inputs, outputs, CODES[dtype], CODES[wide], ps.ACTIVATIONS[activation], 0, 0, 0)))
    most = 0
    for dtype in (torch.bfloat16, torch.float16):
        for wide in (dtype, torch.float32):
            assert ps.Context.linear_backward_bytes(tokens, inputs, outputs, activation, wide) == needed(dtype, wide) > 0
            most = max(most, needed(dtype, wide))
    assert ps.Context.linear_backward_bytes(tokens, inputs, outputs, activation) == most


@pytest.mark.parametrize("dtype", CODES)
@pytest.mark.parametrize("rows, cols", [(1, 1), (300, 64), (4000, 5003), (500, 12000), (300, 70000)])
def test_norm_buffer_is_large_enough(dtype, rows, cols):
    for wide in CODES:
        need = ps._lib.ps_layer_norm_backward_bytes(C.byref(NormDesc(rows, cols, 0.0, CODES[dtype], CODES[wide], 0, 0)))
        assert ps.Context.layer_norm_backward_bytes(rows, cols, dtype) == need > 0
