"""What the exact gradients of tests/test_gpu_mx_exact.py can tell, on the CPU: a bf16 part of dy that is lost shows in every result
that it belongs to, and every step of 64 of either sum has something to lose."""
import pytest
import torch

from tests.test_gpu_mx_exact import CHOSEN, FORMS, NARROW, full, only, operands, places, some

PARTS = {torch.float32: 3, torch.bfloat16: 1, torch.float16: 2}


def parts(v):
    """v as a sum of bf16 numbers, leading bits first."""
    rest, out = v.float(), []
    for _ in range(PARTS[v.dtype]):
        out.append((rest.view(torch.int32) & -65536).view(torch.float32))
        rest = rest - out[-1]
    assert not rest.any()
    return [p.double() for p in out]


@pytest.mark.parametrize("dtype", list(PARTS))
def test_every_part_shows(dtype):
    dy, w = full(1, 40, 70, dtype), some(2, 70, 50)
    for d, a in ((dy, only(w, places(70, 50, 1))), (only(dy.t().contiguous(), places(70, 40, 1)).t().contiguous(), w)):
        want = d.double() @ a.double()
        assert want.all() and torch.equal(want.to(dtype).double(), want)
        for i, lost in enumerate(parts(d)):
            had = lost @ a.double() != 0
            assert had.all() if i == 0 else had.any()       # (16 bits whose first eight are zero are one part)
            assert ((d.double() - lost) @ a.double()).to(dtype).double()[had].ne(want[had]).all()


@pytest.mark.parametrize("rows,c_in,c_out", FORMS + NARROW + CHOSEN)
def test_every_step_has_something_to_lose(rows, c_in, c_out):
    steps_x, steps_w = torch.zeros(-(-c_out // 64)), torch.zeros(-(-rows // 64))
    for turn in range(3):
        for d, a, b in operands(rows, c_in, c_out, torch.float32, turn):
            if a is not None:
                used = (d != 0).any(dim=0) & (a != 0).any(dim=1)
                steps_x[torch.nonzero(used).flatten() // 64] += 1
            if b is not None:
                used = (d != 0).any(dim=1) & (b != 0).any(dim=1)
                steps_w[torch.nonzero(used).flatten() // 64] += 1
    assert steps_x.all() and steps_w.all()
