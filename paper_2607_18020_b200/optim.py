"""Orthogonalised updates of weight matrices.

    X = orthogonalize(G)                               Newton-Schulz iteration on a matrix or a stack of them
    muon_step(weight, grad, momentum, lr=...)          the optimiser's whole step, in place
    Muon(params, lr=...)                               torch.optim.Optimizer over muon_step

Everything runs in libfpde.so on torch's current stream; there is no CPU path.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as B_
from .autograd import ValuesOnly, wants_grad


def _matrices(name, t):
    """`t` as (count, rows, cols)."""
    if t.device.type != "cuda":
        raise ValueError("%s is on %s, expected a CUDA tensor" % (name, t.device))
    if str(t.dtype) not in B_.DTYPE_IDS:
        raise ValueError("%s is %s, expected fp32, bf16 or fp16" % (name, t.dtype))
    if t.dim() not in (2, 3):
        raise ValueError("%s has %d axes, expected a matrix or a stack of matrices" % (name, t.dim()))
    return t.unsqueeze(0) if t.dim() == 2 else t


_plans = B_.ArgPlans()
_lay = _plans.layout


def _args(grad, steps, eps):
    """The argument block of a call without its pointers, and grad with contiguous columns."""
    g = _matrices("grad", grad)
    if g.stride(2) != 1 and g.shape[2] > 1:
        g = g.contiguous()
    a = B_.OrthoArgs(dtype=B_.DTYPE_IDS[str(g.dtype)], steps=steps, count=g.shape[0], rows=g.shape[1], cols=g.shape[2], grad_matrix=g.stride(0),
                     grad_row=g.stride(1), eps=eps)
    a.workspace_bytes = B_.lib().fpde_orthogonalize_workspace_bytes(ctypes.byref(a))
    return a, g


def _plan(name, grad, steps, eps):
    eps = float(eps)                            # a tensor may hold another number in the next call
    key = (name, steps, eps, _lay(grad))
    a = _plans.get(key)
    if a is None:
        a, g = _args(grad, steps, eps)
        if g.data_ptr() == grad.data_ptr():     # a view at most
            _plans.keep(key, a)
        return a, g
    return a, grad


def orthogonalize(grad, steps=5, eps=1e-7):
    """grad (rows, cols), or a stack (count, rows, cols) treated matrix by matrix, with its singular values driven
    towards one: X = grad / (|grad| + eps), then `steps` times X <- a X + (b S + c S S) X with S = X X^T and
    (a, b, c) = (3.4445, -4.775, 2.0315), on the shorter side.  Returns a dense tensor of grad's type.  Not
    differentiable: a backward pass that reaches the result raises."""
    if wants_grad(grad):
        return ValuesOnly.apply(orthogonalize, grad, steps, eps)
    a, g = _plan("ortho", grad, steps, eps)
    dev = grad.device
    out = torch.empty_like(grad) if grad.is_contiguous() else torch.empty(grad.shape, dtype=grad.dtype, device=dev)
    a.grad, a.out = g.data_ptr(), out.data_ptr()
    if a.workspace_bytes:
        ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=dev)
        a.workspace = ws.data_ptr()
    B_.call_with("fpde_orthogonalize", a, dev.index)
    return out


def muon_step(weight, grad, momentum, lr, momentum_decay=0.95, weight_decay=0.0, nesterov=True, steps=5, eps=1e-7):
    """One step of the optimiser on a matrix or a stack of equal matrices, in place on weight and momentum:

        momentum <- momentum_decay * momentum + grad
        weight   <- (1 - lr * weight_decay) * weight - lr * sqrt(max(1, rows / cols)) * orthogonalize(update)

    where update is grad + momentum_decay * momentum (nesterov) or momentum.  weight and grad have one type,
    momentum is fp32."""
    if grad.shape != weight.shape or momentum.shape != weight.shape:
        raise ValueError("weight %s, grad %s and momentum %s differ in shape" % (tuple(weight.shape), tuple(grad.shape), tuple(momentum.shape)))
    if grad.dtype != weight.dtype or momentum.dtype != torch.float32:
        raise ValueError("grad must have weight's type and momentum be fp32")
    if grad.device != weight.device or momentum.device != weight.device:
        raise ValueError("weight, grad and momentum live on different devices")
    if not (weight.is_contiguous() and momentum.is_contiguous()):
        raise ValueError("weight and momentum are updated in place and must be contiguous")
    a, g = _plan("muon", grad, steps, eps)
    dev = weight.device
    a.nesterov = int(nesterov)
    a.grad, a.weight, a.momentum = g.data_ptr(), weight.data_ptr(), momentum.data_ptr()
    if a.workspace_bytes:
        ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=dev)
        a.workspace = ws.data_ptr()
    a.lr, a.momentum_decay, a.weight_decay = lr, momentum_decay, weight_decay
    B_.call_with("fpde_muon_step", a, dev.index)
    torch.autograd.graph.increment_version((weight, momentum))    # they changed behind autograd's back


class Muon(torch.optim.Optimizer):
    """muon_step over parameters that are matrices or stacks of matrices (give vectors and the input and output
    layers to another optimiser).  The momentum is kept in fp32 whatever the parameters' type."""

    def __init__(self, params, lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, eps=1e-7):
        if lr < 0 or not 0 <= momentum < 1 or weight_decay < 0 or steps < 0 or eps < 0:
            raise ValueError("Muon: a setting is outside its range")
        super().__init__(params, dict(lr=lr, momentum=momentum, weight_decay=weight_decay, nesterov=nesterov, steps=steps, eps=eps))
        for group in self.param_groups:
            for p in group["params"]:
                if p.dim() not in (2, 3):
                    raise ValueError("Muon takes matrices and stacks of matrices, got a parameter of shape %s" % (tuple(p.shape),))

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            for p in group["params"]:
                if p.grad is None:
                    continue
                state = self.state[p]
                if "momentum" not in state:
                    state["momentum"] = torch.zeros(p.shape, dtype=torch.float32, device=p.device)
                muon_step(p, p.grad, state["momentum"], lr=group["lr"], momentum_decay=group["momentum"],
                          weight_decay=group["weight_decay"], nesterov=group["nesterov"], steps=group["steps"], eps=group["eps"])
        return loss

    def load_state_dict(self, state_dict):
        """torch's own call casts the state to the parameters' type; the momentum stays fp32."""
        super().load_state_dict(state_dict)
        saved = [i for g in state_dict["param_groups"] for i in g["params"]]
        mine = [p for g in self.param_groups for p in g["params"]]
        for i, p in zip(saved, mine):
            entry = state_dict["state"].get(i)
            if entry is not None:
                self.state[p]["momentum"] = entry["momentum"].detach().to(device=p.device, dtype=torch.float32, copy=True)
