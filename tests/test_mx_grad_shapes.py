"""Blocks whose bytes come to the same as those of another shape (rows filled up to 32, columns to 256 or 32): the layer's
gradients refuse them, compiled path or not, and never take them for what they are not."""
import types

import pytest
import torch

import paper_1801_09449_amd as T
from paper_1801_09449_amd import binding

# dy's shape, w's or None, the checkpoint's or None
WRONG = [((4, 20), (8, 64), None),              # 12 rows of weights that are not there
         ((4, 8), (8, 64), (4, 40)),            # a checkpoint of 40 columns for 64
         ((64, 8), (8, 32), (32, 64)),          # 32 rows of 64 for 64 rows of 32
         ((64, 8), None, (32, 64)),
         ((2, 40), (64, 300), (2, 300))]
RIGHT = [((4, 20), (20, 64), (4, 64)), ((2, 3, 20), (20, 64), (2, 3, 64)), ((2, 3, 20), None, (2, 3, 64)), ((20,), (20, 64), (64,))]


def blocks(shape, kind, device):
    if shape is None:
        return None
    rows = torch.Size(shape[:-1]).numel()
    return T.MxTensor(torch.zeros(T.tern_mx_bytes(rows, shape[-1], kind), dtype=torch.uint8, device=device), kind, shape)


@pytest.fixture
def compiled(monkeypatch):
    """Stands for the compiled path: notes that it was asked, and answers."""
    asked = []
    T.lib()
    monkeypatch.setattr(binding, "_native", types.SimpleNamespace(mx_linear_grad=lambda *a: asked.append(a) or "done"))
    return asked


@pytest.mark.parametrize("dy,w,saved", WRONG)
def test_the_compiled_path_is_not_asked_for_other_shapes(compiled, dy, w, saved):
    with pytest.raises(ValueError):
        T.tern_mx_linear_grad(torch.zeros(dy), blocks(w, "f4", "cpu"), blocks(saved, "i8", "cpu"))
    assert not compiled


@pytest.mark.parametrize("dy,w,saved", RIGHT)
def test_the_compiled_path_is_asked_for_what_fits(compiled, dy, w, saved):
    assert T.tern_mx_linear_grad(torch.zeros(dy), blocks(w, "f4", "cpu"), blocks(saved, "i8", "cpu"), bias=True) == "done"
    assert len(compiled) == 1 and compiled[0][3] == 64 and compiled[0][4] is True


def test_what_is_no_tensor_is_refused_by_name():
    with pytest.raises(TypeError, match="dy"):
        T.tern_mx_linear_grad([1.0], blocks((8, 64), "f4", "cpu"), None)
    with pytest.raises(ValueError):
        T.tern_mx_linear_grad(torch.zeros(()), blocks((8, 64), "f4", "cpu"), None)


@pytest.mark.gpu
@pytest.mark.parametrize("built", [True, False], ids=["compiled", "ctypes"])
@pytest.mark.parametrize("dy,w,saved", WRONG)
def test_blocks_of_another_shape_are_refused(monkeypatch, built, dy, w, saved):
    T.lib()
    if not built:
        monkeypatch.setattr(binding, "_native", False)
    with pytest.raises(ValueError):
        T.tern_mx_linear_grad(torch.zeros(dy, device="cuda"), blocks(w, "f4", "cuda"), blocks(saved, "i8", "cuda"))
