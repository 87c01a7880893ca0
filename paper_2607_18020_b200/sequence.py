"""Sequence operators of a network that marches fields along one axis of the grid: a short causal
convolution and a selective state space scan over rows of (batch, length, channels) tensors.

    y = causal_conv(x, weight, bias)                              differentiable
    y = selective_scan(u, delta, A, B, C, D, z, delta_bias)       differentiable

with `state=` / `return_state=True` for a row that continues an earlier one, and for one node at a time

    y = causal_conv_step(x, window, weight, bias)                 window moved on in place
    y = selective_scan_step(state, u, delta, A, B, C, D, z, ...)  state moved on in place

`*_fwd` / `*_bwd` are the same calls without autograd.  The single-node forms are not differentiable either:
they compute values, and a backward pass that reaches their result raises.  Activations are fp32, bf16 or fp16 CUDA tensors
of one type whose channel axis is contiguous (slices of a wider projection are read in place);
parameters and scan states are fp32.  Everything runs in libfpde.so on torch's current stream; torch
allocates the outputs and the scratch memory.  There is no CPU path.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as B_
from .autograd import ValuesOnly, wants_grad


class ConvGrads(NamedTuple):
    x: torch.Tensor
    weight: torch.Tensor
    bias: Optional[torch.Tensor]
    state: Optional[torch.Tensor]


class ScanGrads(NamedTuple):
    u: torch.Tensor
    delta: torch.Tensor
    A: torch.Tensor
    B: torch.Tensor
    C: torch.Tensor
    D: Optional[torch.Tensor]
    z: Optional[torch.Tensor]
    delta_bias: Optional[torch.Tensor]
    state: Optional[torch.Tensor]


def _activation(name, t, shape, dtype, device):
    """`t` with a contiguous last axis; checked against what the call expects."""
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype != dtype:
        raise ValueError("%s is %s, expected %s" % (name, t.dtype, dtype))
    if t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))
    return t if t.stride(-1) == 1 or t.shape[-1] <= 1 else t.contiguous()


def _dense(name, t, shape, dtype, device):
    if t is None:
        return None
    _activation(name, t, shape, dtype, device)
    return t.contiguous()


def _same(given, taken):
    return all(a is b for a, b in zip(given, taken))


def _first(name, t, dims):
    if t.device.type != "cuda":
        raise ValueError("%s is on %s, expected a CUDA tensor" % (name, t.device))
    if str(t.dtype) not in B_.DTYPE_IDS:
        raise ValueError("%s is %s, expected fp32, bf16 or fp16" % (name, t.dtype))
    if t.dim() != dims:
        raise ValueError("%s has %d axes, expected %d" % (name, t.dim(), dims))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _new(like, shape=None):
    """A dense tensor of `like`'s type, shape (or `shape`) and device."""
    if like is None:
        return None
    if shape is None and like.is_contiguous():
        return torch.empty_like(like)            # a third of empty()'s host time
    return torch.empty(like.shape if shape is None else shape, dtype=like.dtype, device=like.device)


# For a tensor changed behind autograd's back: a backward pass that has kept it must not take it for what it was.
_moved_on = torch.autograd.graph.increment_version


_plans = B_.ArgPlans()
_lay = _plans.layout


# ------------------------------------------------------------------------------------- convolution
def _conv_args(x, weight, bias, state, silu, step, gy=None, gstate=None, workspace=False):
    """The argument block of a convolution call without its pointers, and the tensors as the call takes them:
    checked, with contiguous channels, parameters and states dense."""
    _first("x", x, 2 if step else 3)
    dev, dt = x.device, x.dtype
    batch, channels = x.shape[0], x.shape[-1]
    if weight.dim() != 2:
        raise ValueError("weight has %d axes, expected 2 (channels, width)" % weight.dim())
    width = weight.shape[1]
    window = (batch, width - 1, channels)
    x = _activation("x", x, x.shape, dt, dev)
    weight = _dense("weight", weight, (channels, width), torch.float32, dev)
    bias = _dense("bias", bias, (channels,), torch.float32, dev)
    if step:
        _activation("window", state, window, dt, dev)
        if not state.is_contiguous():
            raise ValueError("window is updated in place and must be contiguous")
    else:
        state = _dense("state", state, window, dt, dev)
    a = B_.ConvArgs(dtype=B_.DTYPE_IDS[str(dt)], width=width, silu=int(silu), batch=batch, length=1 if step else x.shape[1], channels=channels,
                    x_batch=x.stride(0), x_node=0 if step else x.stride(1))
    if gy is not None:
        gy = _activation("gy", gy, x.shape, dt, dev)
        a.gy_batch, a.gy_node = gy.stride(0), gy.stride(1)
    gstate = _dense("gstate", gstate, window, dt, dev)
    if workspace:
        a.workspace_bytes = B_.lib().fpde_causal_conv_workspace_bytes(ctypes.byref(a))
    return a, (x, weight, bias, state, gy, gstate)


def causal_conv_fwd(x, weight, bias=None, state=None, silu=True):
    """y[t] = act(bias + sum_j weight[:, j] x[t - width + 1 + j]) along axis 1 of x (batch, length, channels), and
    the window (batch, width - 1, channels) that the next call continues from.  Before node 0 stands `state`,
    such a window of an earlier call, or zeros.  weight: (channels, width), width 1 to 4; bias: (channels)."""
    key = ("conv fwd", bool(silu), _lay(x), _lay(weight), _lay(bias), _lay(state))
    a = _plans.get(key)
    if a is None:
        given = (x, weight, bias, state)
        a, (x, weight, bias, state, _, _) = _conv_args(x, weight, bias, state, silu, False)
        if _same(given, (x, weight, bias, state)):
            _plans.keep(key, a)
    dev = x.device
    y = _new(x)
    left = _new(x, (a.batch, a.width - 1, a.channels)) if state is None else _new(state)
    a.x, a.weight, a.bias, a.state = x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(state)
    a.y, a.state_out = y.data_ptr(), left.data_ptr()
    B_.call_with("fpde_causal_conv_fwd", a, dev.index)
    return y, left


def causal_conv_bwd(gy, x, weight, bias=None, state=None, silu=True, gstate=None) -> ConvGrads:
    """Gradients of causal_conv_fwd for upstream gradients gy of y and `gstate` of the window it left."""
    key = ("conv bwd", bool(silu), _lay(gy), _lay(x), _lay(weight), _lay(bias), _lay(state), _lay(gstate))
    a = _plans.get(key)
    if a is None:
        given = (x, weight, bias, state, gy, gstate)
        a, taken = _conv_args(x, weight, bias, state, silu, False, gy, gstate, True)
        if _same(given, taken):
            _plans.keep(key, a)
        x, weight, bias, state, gy, gstate = taken
    dev = x.device
    gx, gw, gb, gs = _new(x), _new(weight), _new(bias), _new(state)
    ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=dev)
    a.x, a.weight, a.bias, a.state = x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(state)
    a.gy, a.gstate_out, a.gx, a.gstate = gy.data_ptr(), _ptr(gstate), gx.data_ptr(), _ptr(gs)
    a.gweight, a.gbias, a.workspace = gw.data_ptr(), _ptr(gb), ws.data_ptr()
    B_.call_with("fpde_causal_conv_bwd", a, dev.index)
    return ConvGrads(gx, gw, gb, gs)


def causal_conv_step(x, window, weight, bias=None, silu=True):
    """One node per row: x (batch, channels) -> y; `window` (batch, width - 1, channels) is moved on in place.
    Not differentiable."""
    if torch.is_grad_enabled() and wants_grad(x, window, weight, bias):
        return ValuesOnly.apply(causal_conv_step, x, window, weight, bias, silu)
    key = ("conv step", bool(silu), _lay(x), _lay(window), _lay(weight), _lay(bias))
    a = _plans.get(key)
    if a is None:
        given = (x, weight, bias)
        a, (x, weight, bias, _, _, _) = _conv_args(x, weight, bias, window, silu, True)
        if _same(given, (x, weight, bias)):
            _plans.keep(key, a)
    y = _new(x)
    a.x, a.weight, a.bias, a.y = x.data_ptr(), weight.data_ptr(), _ptr(bias), y.data_ptr()
    a.state = a.state_out = window.data_ptr()
    B_.call_with("fpde_causal_conv_step", a, x.device.index)
    _moved_on(window)
    return y


class _CausalConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, state, silu):
        y, left = causal_conv_fwd(x, weight, bias, state, silu)
        ctx.save_for_backward(x, weight, bias, state)
        ctx.silu = silu
        ctx.set_materialize_grads(False)
        return y, left

    @staticmethod
    @once_differentiable
    def backward(ctx, gy, gleft):
        x, weight, bias, state = ctx.saved_tensors
        if gy is None:
            gy = torch.zeros_like(x)
        g = causal_conv_bwd(gy, x, weight, bias, state, ctx.silu, gleft)
        return g.x, g.weight, g.bias, g.state, None


def causal_conv(x, weight, bias=None, state=None, silu=True, return_state=False):
    """causal_conv_fwd, differentiable in x, weight, bias and state."""
    y, left = _CausalConv.apply(x, weight, bias, state, silu)
    return (y, left) if return_state else y


# -------------------------------------------------------------------------------------------- scan
def _scan_args(u, delta, A, B, C, D, z, delta_bias, delta_softplus, state, step, gout=None, gstate=None, keep=False, backward=False):
    """As _conv_args, for a scan call."""
    _first("u", u, 2 if step else 3)
    dev, dt, lead, channels = u.device, u.dtype, u.shape[:-1], u.shape[-1]
    if A.dim() != 2:
        raise ValueError("A has %d axes, expected 2 (channels, states)" % A.dim())
    states = A.shape[1]
    rest = (u.shape[0], channels, states)
    u = _activation("u", u, u.shape, dt, dev)
    delta = _activation("delta", delta, u.shape, dt, dev)
    z = None if z is None else _activation("z", z, u.shape, dt, dev)
    B = _activation("B", B, lead + (states,), dt, dev)
    C = _activation("C", C, lead + (states,), dt, dev)
    A = _dense("A", A, (channels, states), torch.float32, dev)
    D = _dense("D", D, (channels,), torch.float32, dev)
    delta_bias = _dense("delta_bias", delta_bias, (channels,), torch.float32, dev)
    if step:
        _activation("state", state, rest, torch.float32, dev)
        if not state.is_contiguous():
            raise ValueError("state is updated in place and must be contiguous")
    else:
        state = _dense("state", state, rest, torch.float32, dev)
    a = B_.ScanArgs(dtype=B_.DTYPE_IDS[str(dt)], states=states, softplus=int(delta_softplus), batch=u.shape[0], length=1 if step else u.shape[1],
                    channels=channels, u_batch=u.stride(0), delta_batch=delta.stride(0), B_batch=B.stride(0), C_batch=C.stride(0))
    if z is not None:
        a.z_batch = z.stride(0)
    if not step:
        a.u_node, a.delta_node, a.B_node, a.C_node = u.stride(1), delta.stride(1), B.stride(1), C.stride(1)
        if z is not None:
            a.z_node = z.stride(1)
        if gout is not None:
            gout = _activation("gout", gout, u.shape, dt, dev)
            a.gout_batch, a.gout_node = gout.stride(0), gout.stride(1)
        gstate = _dense("gstate", gstate, rest, torch.float32, dev)
        if keep:
            a.kept_bytes = B_.lib().fpde_selective_scan_kept_bytes(ctypes.byref(a))
        a.workspace_bytes = B_.lib().fpde_selective_scan_workspace_bytes(ctypes.byref(a), int(backward))
    return a, (u, delta, A, B, C, D, z, delta_bias, state, gout, gstate)


def _scan_pointers(a, u, delta, A, B, C, D, z, delta_bias, state):
    a.u, a.delta, a.A, a.B, a.C = u.data_ptr(), delta.data_ptr(), A.data_ptr(), B.data_ptr(), C.data_ptr()
    a.D, a.z, a.delta_bias, a.state = _ptr(D), _ptr(z), _ptr(delta_bias), _ptr(state)


def selective_scan_fwd(u, delta, A, B, C, D=None, z=None, delta_bias=None, delta_softplus=True, state=None, keep=False):
    """The scan of each row of u (batch, length, channels):

        dt = softplus(delta + delta_bias);  h[t] = exp(dt A) h[t-1] + dt B[t] u[t];  out[t] = (C[t].h[t] + D u[t]) * silu(z[t])

    with A (channels, states), B and C (batch, length, states), h[-1] = state (batch, channels, states) or zeros;
    D, z, delta_bias and the softplus may be left out.  Returns (out, the last state, what selective_scan_bwd
    needs of this pass if `keep`, else None).  1 to 64 states."""
    t = (u, delta, A, B, C, D, z, delta_bias, state)
    key = ("scan fwd", bool(delta_softplus), bool(keep), _lay(u), _lay(delta), _lay(A), _lay(B), _lay(C), _lay(D), _lay(z), _lay(delta_bias),
           _lay(state))
    a = _plans.get(key)
    if a is None:
        a, taken = _scan_args(*t[:8], delta_softplus, state, False, keep=keep)
        if _same(t, taken):
            _plans.keep(key, a)
        t = taken[:9]
    dev = u.device
    out = _new(u)
    last = _new(A, (a.batch, a.channels, a.states)) if state is None else _new(state)
    _scan_pointers(a, *t)
    a.out, a.state_out = out.data_ptr(), last.data_ptr()
    kept = None
    if keep:
        kept = torch.empty(a.kept_bytes, dtype=torch.uint8, device=dev)
        a.kept = kept.data_ptr()
    if a.workspace_bytes:
        ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=dev)
        a.workspace = ws.data_ptr()
    B_.call_with("fpde_selective_scan_fwd", a, dev.index)
    return out, last, kept


def selective_scan_bwd(gout, u, delta, A, B, C, D=None, z=None, delta_bias=None, delta_softplus=True, state=None, kept=None,
                       gstate=None) -> ScanGrads:
    """Gradients of selective_scan_fwd (called with keep=True: pass its `kept`) for upstream gradients gout of
    `out` and `gstate` of the last state."""
    if kept is None:
        raise ValueError("selective_scan_bwd needs what selective_scan_fwd(..., keep=True) returned")
    t = (u, delta, A, B, C, D, z, delta_bias, state, gout, gstate)
    key = ("scan bwd", bool(delta_softplus), _lay(u), _lay(delta), _lay(A), _lay(B), _lay(C), _lay(D), _lay(z), _lay(delta_bias), _lay(state),
           _lay(gout), _lay(gstate))
    a = _plans.get(key)
    if a is None:
        a, taken = _scan_args(*t[:8], delta_softplus, state, False, gout, gstate, backward=True)
        if _same(t, taken):
            _plans.keep(key, a)
        t = taken
    dev = u.device
    if kept.device != dev:
        raise ValueError("kept is on %s, expected %s" % (kept.device, dev))
    g = ScanGrads(_new(u), _new(delta), _new(A), _new(B), _new(C), _new(D), _new(z), _new(delta_bias), _new(state))
    _scan_pointers(a, *t[:9])
    a.gout, a.gstate_out = t[9].data_ptr(), _ptr(t[10])
    a.gu, a.gdelta, a.gA, a.gB, a.gC = g.u.data_ptr(), g.delta.data_ptr(), g.A.data_ptr(), g.B.data_ptr(), g.C.data_ptr()
    a.gD, a.gz, a.gdelta_bias, a.gstate = _ptr(g.D), _ptr(g.z), _ptr(g.delta_bias), _ptr(g.state)
    a.kept, a.kept_bytes = kept.data_ptr(), kept.numel() * kept.element_size()
    ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=dev)
    a.workspace = ws.data_ptr()
    B_.call_with("fpde_selective_scan_bwd", a, dev.index)
    return g


def selective_scan_step(state, u, delta, A, B, C, D=None, z=None, delta_bias=None, delta_softplus=True):
    """One node per row: u, delta, z (batch, channels), B, C (batch, states) -> out (batch, channels); `state`
    (batch, channels, states) is moved on in place.  Not differentiable."""
    t = (u, delta, A, B, C, D, z, delta_bias, state)
    if torch.is_grad_enabled() and wants_grad(*t):
        return ValuesOnly.apply(selective_scan_step, state, u, delta, A, B, C, D, z, delta_bias, delta_softplus)
    key = ("scan step", bool(delta_softplus), _lay(u), _lay(delta), _lay(A), _lay(B), _lay(C), _lay(D), _lay(z), _lay(delta_bias), _lay(state))
    a = _plans.get(key)
    if a is None:
        a, taken = _scan_args(*t[:8], delta_softplus, state, True)
        if _same(t, taken):
            _plans.keep(key, a)
        t = taken[:9]
    out = _new(u)
    _scan_pointers(a, *t)
    a.state_out, a.out = state.data_ptr(), out.data_ptr()
    B_.call_with("fpde_selective_scan_step", a, u.device.index)
    _moved_on(state)
    return out


class _SelectiveScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, delta, A, B, C, D, z, delta_bias, delta_softplus, state, keep):
        out, last, kept = selective_scan_fwd(u, delta, A, B, C, D, z, delta_bias, delta_softplus, state, keep)
        ctx.save_for_backward(u, delta, A, B, C, D, z, delta_bias, state, kept)
        ctx.delta_softplus = delta_softplus
        ctx.set_materialize_grads(False)
        return out, last

    @staticmethod
    @once_differentiable
    def backward(ctx, gout, glast):
        u, delta, A, B, C, D, z, delta_bias, state, kept = ctx.saved_tensors
        if gout is None:
            gout = torch.zeros_like(u)
        g = selective_scan_bwd(gout, u, delta, A, B, C, D, z, delta_bias, ctx.delta_softplus, state, kept, glast)
        return g.u, g.delta, g.A, g.B, g.C, g.D, g.z, g.delta_bias, None, g.state, None


def selective_scan(u, delta, A, B, C, D=None, z=None, delta_bias=None, delta_softplus=True, state=None, return_state=False):
    """selective_scan_fwd, differentiable in every tensor."""
    # decided here: inside forward() grad mode is always off, and parameters ask for gradients in any mode
    keep = wants_grad(u, delta, A, B, C, D, z, delta_bias, state)
    out, last = _SelectiveScan.apply(u, delta, A, B, C, D, z, delta_bias, delta_softplus, state, keep)
    return (out, last) if return_state else out
