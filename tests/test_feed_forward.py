"""The gated block's autograd on the CPU, with float stand-ins for the library's calls (blocks hold the values themselves):
what it hands out, what it refuses to derive, and what it keeps for how long."""
import gc
import weakref

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_1801_09449_amd import binding, feed_forward
from paper_1801_09449_amd.feed_forward import FeedForward


class Floats:
    """The library's calls in floats."""

    def blocks(self, x, kind):
        return binding.MxTensor(x.detach().clone(), kind, x.shape)

    def tern_mx_quantize(self, x, kind="f4"):
        return self.blocks(x, kind)

    def tern_mx_linear(self, x, w, bias=None, save=False):
        x = x.detach()
        y = x @ w.data.t() + (0 if bias is None else bias.detach())
        return (y, self.blocks(x, "i8")) if save else y

    def tern_mx_gate(self, gu, save=False):
        g, u = gu.detach().chunk(2, dim=-1)
        h = torch.nn.functional.silu(g) * u
        return (h, self.blocks(torch.stack([g, u]), "i8")) if save else h

    def tern_mx_linear_grad(self, dy, w, saved, bias=False):
        dy = dy.detach()
        flat = dy.reshape(-1, dy.shape[-1])
        dw = None if saved is None else flat.t() @ saved.data.reshape(-1, saved.data.shape[-1])
        return None if w is None else dy @ w.data, dw, flat.sum(dim=0) if bias else None

    def tern_mx_gate_grad(self, dh, saved, hidden=False):
        g, u = saved.data
        s, dh = torch.sigmoid(g), dh.detach()
        dgu = torch.cat([dh * u * s * (1 + g * (1 - s)), dh * g * s], dim=-1)
        return (dgu, self.blocks(g * s * u, "i8")) if hidden else dgu


@pytest.fixture
def floats(monkeypatch):
    f = Floats()
    monkeypatch.setattr(feed_forward.B, "tern_mx_quantize", f.tern_mx_quantize)
    for name in ("tern_mx_linear", "tern_mx_gate", "tern_mx_linear_grad", "tern_mx_gate_grad"):
        monkeypatch.setattr(feed_forward.B, name, getattr(f, name))
    return f


def block(d=6, c=5, bias=True, grad=True):
    g = torch.Generator().manual_seed(0)
    mk = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).requires_grad_(grad)
    return FeedForward(mk(2 * c, d), mk(d, c), mk(2 * c) if bias else None, mk(d) if bias else None)


def plain(f, x):
    gu = x @ f.w_up.t() + f.b_up
    g, u = gu.chunk(2, dim=-1)
    return (torch.nn.functional.silu(g) * u) @ f.w_down.t() + f.b_down


def test_gradients_are_those_of_the_formula(floats):
    f = block()
    x = torch.randn(2, 3, 6, dtype=torch.float64, requires_grad=True)
    params = [x, f.w_up, f.w_down, f.b_up, f.b_down]
    dy = torch.randn(2, 3, 6, dtype=torch.float64)
    got = torch.autograd.grad(f(x), params, dy)
    for a, b in zip(got, torch.autograd.grad(plain(f, x), params, dy)):
        torch.testing.assert_close(a, b)


@pytest.mark.parametrize("weighted", [False, True], ids=["of a sum", "of a trained sum"])
def test_a_second_derivative_is_refused(floats, weighted):
    # a gradient penalty beside an ordinary term must not train as if it were not there
    f = block()
    x = torch.randn(3, 6, dtype=torch.float64, requires_grad=True)
    by = torch.ones(6, dtype=torch.float64, requires_grad=True) if weighted else 1.0
    with pytest.raises(RuntimeError, match="again"):
        dx, = torch.autograd.grad((f(x) * by).sum(), x, create_graph=True)
        torch.autograd.grad(dx.square().sum() + plain(f, x).sum(), x)
    torch.autograd.grad((f(x) * by).sum(), x)


@pytest.mark.parametrize("grad", [True, False], ids=["grad", "no_grad"])
@pytest.mark.parametrize("which", ["x", "w_up", "w_down", "b_up", "b_down"])
def test_a_forward_mode_derivative_is_refused(floats, which, grad):
    f = block(grad=False)
    x = torch.randn(3, 6, dtype=torch.float64)
    with forward_ad.dual_level(), torch.set_grad_enabled(grad):
        f(x)
        t = x if which == "x" else getattr(f, which)
        dual = forward_ad.make_dual(t, torch.ones_like(t))
        if which == "x":
            x = dual
        else:
            setattr(f, which, dual)
        with pytest.raises(NotImplementedError):
            f(x)
    with pytest.raises(NotImplementedError):
        torch.func.jvp(block(grad=False), (torch.zeros(3, 6, dtype=torch.float64),), (torch.ones(3, 6, dtype=torch.float64),))


def kept_by(floats, monkeypatch):
    """Weak references to the checkpoints that forward passes make from here on."""
    left = []

    def noting(call):
        def noted(*a, **k):
            out = call(*a, **k)
            if k.get("save"):
                left.append(weakref.ref(out[1].data))
            return out
        return noted
    for name in ("tern_mx_linear", "tern_mx_gate"):
        monkeypatch.setattr(feed_forward.B, name, noting(getattr(floats, name)))
    return left


def test_the_checkpoint_goes_with_its_backward_pass(floats, monkeypatch):
    left = kept_by(floats, monkeypatch)
    f = block()
    loss = f(torch.randn(3, 6, dtype=torch.float64)).sum()
    gc.collect()
    assert len(left) == 2 and all(r() is not None for r in left)
    loss.backward()
    gc.collect()
    assert all(r() is None for r in left)       # though the loss, and its graph, are still there
    with pytest.raises(RuntimeError):
        loss.backward()                         # as every other layer says a second time
    loss = f(torch.randn(3, 6, dtype=torch.float64)).sum()
    f.w_up.grad = None
    loss.backward(retain_graph=True)
    once, f.w_up.grad = f.w_up.grad, None
    loss.backward()
    assert torch.equal(f.w_up.grad, once)


def test_hooks_on_what_is_saved_see_the_checkpoint(floats):
    f = block()
    x = torch.randn(3, 6, dtype=torch.float64)
    want = torch.autograd.grad(f(x).sum(), f.w_up)[0]
    packed = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: packed.append(t.clone()) or len(packed) - 1, lambda i: packed[i]):
        y = f(x)
    shapes = [tuple(t.shape) for t in packed]
    assert (3, 6) in shapes and (2, 3, 5) in shapes
    assert torch.equal(torch.autograd.grad(y.sum(), f.w_up)[0], want)
