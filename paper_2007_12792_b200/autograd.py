"""The physics loss as a differentiable PyTorch op: forward = per-sample energies J from the fused
CUDA kernel, backward = the residual the same kernel produced (the loss gradient that enters the
generator's back-propagation in Algorithm 1).  No autograd graph is built inside; there is no CPU path.

Also two layers of a generator that the losses are back-propagated through: the gated recurrence over the time rows of
a field, and pointwise activations, both able to keep what their backward pass needs in 8 bits (``checkpoints``
does the same for the saved tensors of any other op, these losses' gradients among them)."""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import binding as B
from . import checkpoints


def _apply(name, where, function, u, problem, workspace):
    """The loss as a native autograd function; arguments it does not recognise go to the one below, with its errors."""
    loss = getattr(B.native(), name)(u, problem, workspace)
    if isinstance(loss, torch.Tensor):
        return loss
    if loss is not None:
        raise B.DnError(loss, where)
    return function.apply(u, problem, workspace)


class _Energy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, problem, workspace):
        u = u.contiguous()
        J = torch.empty(problem.batch, dtype=torch.float32, device=u.device)
        r = torch.empty_like(u)
        B.dn_energy_grad(problem, u, None, J, r, workspace)
        ctx.save_for_backward(r)
        return J

    @staticmethod
    def backward(ctx, grad_J):
        (r,) = ctx.saved_tensors
        shape = (-1,) + (1,) * (r.dim() - 1)
        return grad_J.reshape(shape).to(r.dtype) * r, None, None


def energy(u: torch.Tensor, problem: B.Problem, workspace: torch.Tensor = None) -> torch.Tensor:
    """J[b] for a batch of fields u (contiguous float32 CUDA tensor); differentiable with respect to u.
    The gradient is the masked residual K(nu) u - F, so Dirichlet nodes receive zero gradient."""
    if workspace is None:
        workspace = B.new_workspace(problem)
    return _apply("energy_loss", "dn_energy_grad", _Energy, u, problem, workspace)


class _BurgersLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, problem, workspace):
        u = u.contiguous()
        L = torch.empty(problem.batch, dtype=torch.float32, device=u.device)
        g = torch.empty_like(u)
        B.dn_burgers_loss_grad(problem, u, None, L, None, g, workspace)
        ctx.save_for_backward(g)
        return L

    @staticmethod
    def backward(ctx, grad_L):
        (g,) = ctx.saved_tensors
        return grad_L.reshape(-1, 1, 1).to(g.dtype) * g, None, None


def burgers_loss(u: torch.Tensor, problem: B.Burgers, workspace: torch.Tensor = None) -> torch.Tensor:
    """L[b] = L_p + lambda L_b of the Burgers finite-difference loss for a batch of fields u [B][nt][nx]
    (contiguous float32 CUDA tensor); differentiable with respect to u."""
    if workspace is None:
        workspace = B.new_burgers_workspace(problem)
    return _apply("burgers_loss", "dn_burgers_loss_grad", _BurgersLoss, u, problem, workspace)


def gated_scan(gate: torch.Tensor, x: torch.Tensor, h0: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
               mix: bool = False, checkpoint: Optional[str] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(h, h_last) of the recurrence h_t = a_t h_{t-1} + w_t x_t over the rows of fields [batch, rows, cols], a = sigmoid(gate),
    w = 1 or, with ``mix``, 1 - a; h0 and h_last: [batch, cols] float32; lengths: [batch] int32, rows behind them are 0.
    gate and x: CUDA tensors of one type (float32, bfloat16, float16).  Differentiable once, backward, with respect to gate, x and h0.

    checkpoint None keeps gate, x and the state ahead of every 64th row for the backward pass; "int8" or "e4m3" keeps gate and x
    in 8 bits instead (the gate as int8 in either, held to +-63.5), and the gradients are those at the values that 8 bits hold."""
    kept = B._format(checkpoint, none=True)
    checkpoints.saving.gate = checkpoint is None
    try:
        out = B.native().gated_scan(gate, x, h0, lengths, mix, kept)
    finally:
        checkpoints.saving.gate = False
    if isinstance(out, int):
        raise B.DnError(out, "dn_scan_forward")
    return out


def activation(x: torch.Tensor, kind: str = "silu", checkpoint: str = "int8") -> torch.Tensor:
    """"silu", "gelu" (its tanh form) or "tanh" of a CUDA tensor, which keeps its input for the backward pass in 8 bits ("int8" or
    "e4m3"): the gradient is dy f'(x) at the values that 8 bits hold.  Differentiable once, backward."""
    y = B.native().activation(x, B._kind(kind), B._format(checkpoint))
    if isinstance(y, int):
        raise B.DnError(y, "dn_activation_forward")
    return y
