"""A gated feed-forward block on block-scaled numbers: y = (silu(x G^T + a) * (x U^T + b)) D^T + c, its products on
4-bit numbers, trained through 8-bit checkpoints.

The float weights are the caller's (as the paper keeps full-precision weights beside the quantised ones and quantises
before each forward pass); pack() turns them into 4 bits, once for serving and after every optimiser
step in training.  What a training step keeps for its backward pass is x and both halves of the hidden layer in 8 bits:
33/32 bytes a value, where a float16 or bfloat16 layer keeps two for each of them and for the product of the halves.
Gradients are of first order and of backward mode: a backward pass with create_graph=True is an error, and so is a call on
tensors with forward-mode tangents.
"""
from typing import Optional

import torch
import torch.autograd.forward_ad as forward_ad

from . import binding as B


class _Step(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_up, w_down, b_up, b_down, up, down):
        gu, x8 = B.tern_mx_linear(x, up, b_up, save=True)
        h, halves = B.tern_mx_gate(gu, save=True)
        kept = (up, down, x8, halves)                # of this forward pass, whatever is packed later
        ctx.save_for_backward(*(q.data for q in kept))          # (autograd lets go of them with the backward pass)
        ctx.blocks = [(q.kind, q.shape) for q in kept]
        ctx.types = [None if t is None else t.dtype for t in (w_up, w_down, b_up, b_down)]
        return B.tern_mx_linear(h, down, b_down)

    @staticmethod
    def backward(ctx, dy):
        # (a decorator that lets only a derivative of the results fail stays silent where dy is a constant)
        if torch.is_grad_enabled():
            raise RuntimeError("the block's gradients cannot be differentiated again (create_graph=True)")
        up, down, x8, halves = (B.MxTensor(t, *of) for t, of in zip(ctx.saved_tensors, ctx.blocks))
        need_x, need_up, need_down, need_b_up, need_b_down = ctx.needs_input_grad[:5]
        dy = dy.contiguous()
        dx = dw_up = dw_down = db_up = db_down = None
        if need_x or need_up or need_b_up or need_down:
            dh, _, db_down = B.tern_mx_linear_grad(dy, down, None, bias=need_b_down)
            dgu = B.tern_mx_gate_grad(dh, halves, hidden=need_down)
            if need_down:
                dgu, h8 = dgu
                dw_down = B.tern_mx_linear_grad(dy, None, h8)[1]
            if need_x or need_up or need_b_up:
                dx, dw_up, db_up = B.tern_mx_linear_grad(dgu, up if need_x else None, x8 if need_up else None, bias=need_b_up)
        elif need_b_down:
            db_down = B.tern_mx_linear_grad(dy, None, None, bias=True)[2]
        grads = [None if g is None else g.to(t) for g, t in zip((dw_up, dw_down, db_up, db_down), ctx.types)]
        return (dx, *grads, None, None)


class FeedForward:
    """w_up [2 c, d] (rows of G, then of U) and w_down [d, c]: float device tensors, trained by the caller; b_up [2 c] and
    b_down [d]: float32 or None."""

    def __init__(self, w_up: torch.Tensor, w_down: torch.Tensor, b_up: Optional[torch.Tensor] = None,
                 b_down: Optional[torch.Tensor] = None):
        if w_up.dim() != 2 or w_down.dim() != 2 or w_up.shape[0] != 2 * w_down.shape[1] or w_up.shape[1] != w_down.shape[0]:
            raise ValueError("w_up must be [2 c, d] and w_down [d, c]")
        self.w_up, self.w_down, self.b_up, self.b_down = w_up, w_down, b_up, b_down
        self.pack()

    def pack(self) -> None:
        """The float weights as they are now, in 4 bits: what every call from here on multiplies with."""
        with torch.no_grad():
            self.up, self.down = B.tern_mx_quantize(self.w_up, "f4"), B.tern_mx_quantize(self.w_down, "f4")

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        """x [..., d] (float32, bfloat16 or float16; one token or many) -> [..., d].  Keeps what a backward pass needs
        where one may follow."""
        given = (x, self.w_up, self.w_down, self.b_up, self.b_down)
        # (a level is asked for first: five tensors took 2 us of a call)
        if getattr(forward_ad, "_current_level", 0) >= 0 and any(
                t is not None and forward_ad.unpack_dual(t).tangent is not None for t in given):
            raise NotImplementedError("the block has no forward-mode derivative")
        if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in given):
            return _Step.apply(*given, self.up, self.down)
        return B.tern_mx_linear(B.tern_mx_gate(B.tern_mx_linear(x, self.up, self.b_up)), self.down, self.b_down)


def example(steps: int = 40, tokens: int = 512, d: int = 256, c: int = 512, device: str = "cuda"):
    """Trains a block to imitate another one and serves a token with it: (first loss, last loss, the token's output)."""
    g = torch.Generator().manual_seed(0)
    def weights(n, k):
        return (torch.randn(n, k, generator=g) / k ** 0.5).to(device)
    teacher = FeedForward(weights(2 * c, d), weights(d, c))
    block = FeedForward(weights(2 * c, d).requires_grad_(), weights(d, c).requires_grad_(),
                        torch.zeros(2 * c, device=device, requires_grad=True), torch.zeros(d, device=device, requires_grad=True))
    params = [block.w_up, block.w_down, block.b_up, block.b_down]
    optimiser = torch.optim.Adam(params, lr=3e-3)
    x = torch.randn(tokens, d, generator=g).to(device).bfloat16()
    with torch.no_grad():
        target = teacher(x).float()
    losses = []
    for _ in range(steps):
        loss = (block(x).float() - target).square().mean()
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        block.pack()
        losses.append(loss.detach())
    with torch.no_grad():
        token = block(x[:1])
    return float(losses[0]), float(losses[-1]), token


if __name__ == "__main__":
    first, last, token = example()
    print(f"loss {first:.4f} -> {last:.4f}; a token of {tuple(token.shape)}")
