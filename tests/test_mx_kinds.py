"""Kinds and types that there are not are refused by name, before anything is looked at on a GPU."""
import pytest
import torch

import paper_1801_09449_amd as T


@pytest.mark.parametrize("kind", ["f6", "F4", None, 0])
def test_a_kind_that_there_is_not(kind):
    blocks = T.MxTensor(torch.zeros(66, dtype=torch.uint8), kind, (2, 32))
    for call in (lambda: T.tern_mx_quantize(torch.zeros(2, 32), kind), lambda: T.tern_mx_bytes(2, 32, kind), lambda: T.tern_mx_values(blocks)):
        with pytest.raises(KeyError, match="kind must be 'f4' or 'i8'"):
            call()


@pytest.mark.parametrize("dtype", [torch.float64, torch.int8, None])
def test_a_type_that_there_is_not(dtype):
    for call in (lambda: T.tern_mx_linear_grad_workspace_bytes(dtype, 2, 32, 32),
                 lambda: T.tern_mx_values(T.MxTensor(torch.zeros(66, dtype=torch.uint8), "i8", (2, 32)), dtype)):
        with pytest.raises(TypeError, match="dtype must be float32, bfloat16 or float16"):
            call()


def test_what_is_no_tensor():
    halves = T.MxTensor(torch.zeros(132, dtype=torch.uint8), "i8", (2, 2, 32))
    with pytest.raises(TypeError, match="dh"):
        T.tern_mx_gate_grad([1.0], halves)
    with pytest.raises(TypeError, match="gu"):
        T.tern_mx_gate([1.0])
    with pytest.raises(TypeError, match="x"):
        T.tern_mx_quantize([1.0])
    with pytest.raises(TypeError, match="x"):
        T.tern_mx_linear([1.0], T.MxTensor(torch.zeros(4352, dtype=torch.uint8), "f4", (2, 32)))
    with pytest.raises(TypeError, match="q"):
        T.tern_mx_values(None)
