"""Gradients whose sums are exact, so that every bit of dy shows in them: a float's last eight bits (the third of the bf16 numbers
that it is taken as) are far below any bound on rounded sums.

Either every column of the other operand has one number that is not zero, or every row (for dw: column) of dy has; those of
the other operand are powers of two that a block holds as they are.  A result is then a value of dy times a power of
two, whatever the order of its sum, its shares or its waves."""
import pytest
import torch

import paper_1801_09449_amd as T
from tests.test_gpu_mx import TYPES

pytestmark = pytest.mark.gpu
FORM, SPLITS = 9, 10


def full(seed, rows, cols, dtype):
    """Numbers whose significands are as long as the type's, the last bit set."""
    r = torch.Generator().manual_seed(seed)
    bits = {torch.float32: 24, torch.bfloat16: 8, torch.float16: 11}[dtype]
    m = torch.randint(2 ** (bits - 1), 2 ** bits, (rows, cols), generator=r) | 1
    power = torch.randint(-2, 3, (rows, cols), generator=r)
    sign = torch.randint(0, 2, (rows, cols), generator=r) * 2 - 1
    v = (sign * m).double() * torch.exp2((power - bits).double())
    assert torch.equal(v.to(dtype).double(), v)
    return v.to(dtype)


def some(seed, rows, cols):
    """+-1, 2, 4 or 8."""
    r = torch.Generator().manual_seed(seed)
    sign = torch.randint(0, 2, (rows, cols), generator=r) * 2 - 1
    return (sign * 2 ** torch.randint(0, 4, (rows, cols), generator=r)).float()


def only(v, at):
    """v, zero but for row at[j] of column j."""
    keep = torch.zeros_like(v, dtype=torch.bool)
    keep[at, torch.arange(v.shape[1])] = True
    return torch.where(keep, v, torch.zeros((), dtype=v.dtype))


def places(n, count, turn):
    """One of n for each of `count`, from the first to the last of n."""
    if count >= n:
        return (torch.arange(count) + turn) % n
    return ((torch.arange(count) * (n - 1)).div(max(1, count - 1), rounding_mode="floor") + turn) % n


def operands(rows, c_in, c_out, dtype, turn):
    """(dy, w or None, x or None): the three ways in which sums are exact."""
    dy, w, x = full(turn, rows, c_out, dtype), some(10 + turn, c_out, c_in), some(20 + turn, rows, c_in)
    return ((dy, only(w, places(c_out, c_in, turn)), only(x, places(rows, c_in, turn))),
            (only(dy.t().contiguous(), places(c_out, rows, turn)).t().contiguous(), w, None),
            (only(dy, places(rows, c_out, turn)), None, x))


def check(rows, c_in, c_out, dtype):
    for turn in range(3):
        for d, a, b in operands(rows, c_in, c_out, dtype, turn):
            q = None if a is None else T.tern_mx_quantize(a.cuda(), "f4")
            s = None if b is None else T.tern_mx_quantize(b.cuda(), "i8")
            dx, dw, _ = T.tern_mx_linear_grad(d.cuda(), q, s)
            v = d.double().cuda()
            if a is not None:
                assert torch.equal(T.tern_mx_values(q).cpu(), a)
                want = torch.matmul(v, a.double().cuda())
                assert torch.equal(dx.double(), want), f"dx {rows} x {c_in} -> {c_out}, turn {turn}"
            if b is not None:
                assert torch.equal(T.tern_mx_values(s).cpu(), b)
                want = torch.matmul(v.t().contiguous(), b.double().cuda())
                assert torch.equal(dw.double(), want), f"dw {rows} x {c_in} -> {c_out}, turn {turn}"


def forced(form, splits):
    T.tern_set_option(FORM, form)
    T.tern_set_option(SPLITS, splits)


FORMS = [(40, 33, 300), (300, 270, 130), (513, 140, 700), (129, 513, 1030)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form,splits", [(f, s) for f in (1, 2, 3, 4) for s in (1, 3)])
def test_every_form_has_all_bits(form, splits, dtype):
    forced(form, splits)
    try:
        for size in FORMS:
            check(*size, dtype)
    finally:
        forced(0, 0)


# a side of at most 64 (input channels in float and half: 128): one, two, three and four blocks of it, rows of a record's edges
NARROW = [(300, 20, 517), (700, 64, 130), (130, 70, 900), (513, 128, 270),        # dy in rows and down columns
          (20, 300, 700), (64, 517, 260),                                        # the weights
          (517, 300, 20), (700, 130, 63)]                                        # the checkpoint


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("splits", [1, 3, 0])
def test_narrow_layers_have_all_bits(splits, dtype):
    forced(5, splits)
    try:
        for size in NARROW:
            check(*size, dtype)
    finally:
        forced(0, 0)


CHOSEN = [(4100, 40, 4099), (16, 4096, 4100), (4099, 4100, 24), (4100, 100, 8300), (600, 700, 800)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("size", CHOSEN)
def test_what_is_chosen_has_all_bits(size, dtype):
    check(*size, dtype)
