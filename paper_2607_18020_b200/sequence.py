"""Sequence operators of a network that marches fields along one axis of the grid: a short causal
convolution and a selective state space scan over rows of (batch, length, channels) tensors, and linear
attention with a decay for each head over (batch, length, heads, features), with the position rotation
and the norm of its queries and keys.

    y = causal_conv(x, weight, bias)                              differentiable
    y = selective_scan(u, delta, A, B, C, D, z, delta_bias)       differentiable
    q, k = rotary(q, k, inv_freq)                                 differentiable
    q, k = norm_rotary(q, k, q_weight, k_weight, inv_freq)        differentiable
    o = linear_attention(q, k, v, log_decay, scale)               differentiable but in log_decay

with `state=` / `return_state=True` for a row that continues an earlier one, and for one node at a time

    y = causal_conv_step(x, window, weight, bias)                 window moved on in place
    y = selective_scan_step(state, u, delta, A, B, C, D, z, ...)  state moved on in place
    o = linear_attention_step(state, q, k, v, log_decay, scale)   state moved on in place

A row that continues gives the rotation its first node's position: `offset=`, or `positions=` for each row its own.

`*_fwd` / `*_bwd` are the same calls without autograd.  The single-node forms are not differentiable either:
they compute values, and a backward pass that reaches their result raises.  Activations are fp32, bf16 or fp16 CUDA tensors
of one type whose channel or feature axis is contiguous (slices of a wider projection are read in place);
parameters, frequencies and states are fp32.  Everything runs in libfpde.so on torch's current stream; torch
allocates the outputs and the scratch memory.  There is no CPU path.  Calls can be captured into CUDA graphs, a
backward pass as torch allows it: while no eager graph of the same leaves lives.
"""
from __future__ import annotations

import ctypes
import math
import numbers
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


class HeadGrads(NamedTuple):
    q: torch.Tensor
    k: Optional[torch.Tensor]
    q_weight: Optional[torch.Tensor]
    k_weight: Optional[torch.Tensor]


class LinearGrads(NamedTuple):
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
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


def _number(name, x):
    """A setting that a plan is kept by, and so a plain number: a tensor may hold another one in the next call."""
    if type(x) is float:
        return x
    if not isinstance(x, numbers.Real):
        raise ValueError("%s is of type %s, expected a number" % (name, type(x).__name__))
    return float(x)


def _offset(x):
    """A whole number that fits 64 bits: the argument block would take a larger one for what is left of it there."""
    if type(x) is not int and not isinstance(x, numbers.Integral) or not -1 << 63 <= x < 1 << 63:
        raise ValueError("offset is %r, expected a whole number of 64 bits" % (x,))
    return int(x)


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


# ---------------------------------------------------------------------------------- heads and positions
def rotary_frequencies(pairs, base=10000.0, stretch=1.0, length=None, fast=32.0, slow=1.0, device="cuda"):
    """inv_freq (pairs) fp32: pair i turns by base^(-i / pairs) a node, for rows `stretch` times as long as those that a
    network was trained on divided by `stretch`.  With `length`, the nodes of a row in training, pairs that turn more
    than `fast` times over such a row keep their frequency, those under `slow` times are divided, and those between
    are blended."""
    if pairs < 1 or not base > 0 or not stretch > 0 or not 0 < slow < fast:
        raise ValueError("expected pairs >= 1, base > 0, stretch > 0 and 0 < slow < fast")
    freq = base ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
    keep = torch.zeros_like(freq)
    if length is not None:
        keep = ((length * freq / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
    return (freq * (keep + (1 - keep) / stretch)).to(device=device, dtype=torch.float32)


def _heads(a, name, t, dim, dt, dev):
    """A (batch, length, heads, dim) view as the call takes it; its strides go into the argument block."""
    if t.dim() != 4:
        raise ValueError("%s has %d axes, expected 4 (batch, length, heads, features)" % (name, t.dim()))
    t = _activation(name, t, (a.batch, a.length, t.shape[2], dim), dt, dev)
    setattr(a, name + "_batch", t.stride(0))
    setattr(a, name + "_node", t.stride(1))
    setattr(a, name + "_head", t.stride(2))
    return t


def _head_args(norm, q, k, q_weight, k_weight, inv_freq, positions, interleaved, eps, gq=None, gk=None):
    """As _conv_args, for a rotation or norm; without norm the gradients come with gq and gk in the place of q and k."""
    _first("q", q, 4)
    dev, dt, dim = q.device, q.dtype, q.shape[3]
    a = B_.HeadArgs(dtype=B_.DTYPE_IDS[str(dt)], norm=int(norm), interleaved=int(interleaved), batch=q.shape[0], length=q.shape[1], q_heads=q.shape[2],
                    k_heads=0 if k is None else k.shape[2], dim=dim, eps=eps)
    if inv_freq is not None:
        if inv_freq.dim() != 1:
            raise ValueError("inv_freq has %d axes, expected 1 (pairs)" % inv_freq.dim())
        inv_freq = _dense("inv_freq", inv_freq, inv_freq.shape, torch.float32, dev)
        a.pairs = inv_freq.shape[0]
        if 2 * a.pairs > dim:
            raise ValueError("%d pairs do not fit %d features" % (a.pairs, dim))
    if positions is not None:
        if positions.shape != q.shape[:2] or positions.dtype != torch.int64 or positions.device != dev:
            raise ValueError("positions are %s %s on %s, expected int64 %s on %s" % (positions.dtype, tuple(positions.shape), positions.device,
                                                                                    tuple(q.shape[:2]), dev))
        a.pos_batch, a.pos_node = positions.stride()
    q_weight = _dense("q_weight", q_weight, (dim,), torch.float32, dev)
    k_weight = _dense("k_weight", k_weight, (dim,), torch.float32, dev)
    q = _heads(a, "q", q, dim, dt, dev)
    k = None if k is None else _heads(a, "k", k, dim, dt, dev)
    if gq is not None:
        if gq.shape != q.shape or (gk is None) != (k is None) or (gk is not None and gk.shape != k.shape):
            raise ValueError("gq and gk need the shapes of q and k")
        gq = _heads(a, "gq", gq, dim, dt, dev)
        gk = None if gk is None else _heads(a, "gk", gk, dim, dt, dev)
        a.workspace_bytes = B_.lib().fpde_head_rotary_workspace_bytes(ctypes.byref(a))
    return a, (q, k, q_weight, k_weight, inv_freq, positions, gq, gk)


def _head_plan(kind, norm, q, k, q_weight, k_weight, inv_freq, positions, offset, interleaved, eps, gq=None, gk=None):
    eps = _number("eps", eps)
    key = (kind, bool(interleaved), eps, _lay(q), _lay(k), _lay(q_weight), _lay(k_weight), _lay(inv_freq), _lay(positions), _lay(gq), _lay(gk))
    t = (q, k, q_weight, k_weight, inv_freq, positions, gq, gk)
    a = _plans.get(key)
    if a is None:
        a, taken = _head_args(norm, *t[:6], interleaved, eps, gq, gk)
        if _same(t, taken):
            _plans.keep(key, a)
        t = taken
    a.inv_freq, a.positions, a.offset = _ptr(t[4]), _ptr(t[5]), _offset(offset)      # a march has another offset in every call
    return a, t


def _head_fwd(kind, norm, q, k, q_weight, k_weight, inv_freq, positions, offset, interleaved, eps):
    a, t = _head_plan(kind, norm, q, k, q_weight, k_weight, inv_freq, positions, offset, interleaved, eps)
    out_q, out_k = _new(q), _new(k)
    a.q, a.k, a.q_weight, a.k_weight = t[0].data_ptr(), _ptr(t[1]), _ptr(t[2]), _ptr(t[3])
    a.q_out, a.k_out = out_q.data_ptr(), _ptr(out_k)
    B_.call_with("fpde_head_rotary_fwd", a, q.device.index)
    return out_q, out_k


def rotary_fwd(q, k, inv_freq, positions=None, offset=0, interleaved=False):
    """q (batch, length, heads, dim) and k (batch, length, k_heads, dim), or None, with the first 2 * len(inv_freq) features
    of each head turned: pair i, which is (x[i], x[i + pairs]), or interleaved (x[2i], x[2i + 1]), by the angle
    position * inv_freq[i].  The position is offset + t, or offset + positions[b, t] (int64); offset is a whole number of 64 bits."""
    return _head_fwd("rotary fwd", False, q, k, None, None, inv_freq, positions, offset, interleaved, 0.0)


def rotary_bwd(gq, gk, inv_freq, positions=None, offset=0, interleaved=False):
    """Gradients of rotary_fwd in q and k, for upstream gradients gq and gk (or None): turned back."""
    a, t = _head_plan("rotary bwd", False, gq, gk, None, None, inv_freq, positions, offset, interleaved, 0.0)
    out_q, out_k = _new(gq), _new(gk)
    a.gq, a.gq_batch, a.gq_node, a.gq_head = t[0].data_ptr(), a.q_batch, a.q_node, a.q_head
    a.gk, a.gk_batch, a.gk_node, a.gk_head = _ptr(t[1]), a.k_batch, a.k_node, a.k_head
    a.gx_q, a.gx_k = out_q.data_ptr(), _ptr(out_k)
    B_.call_with("fpde_head_rotary_bwd", a, gq.device.index)
    return out_q, out_k


def norm_rotary_fwd(q, k, q_weight=None, k_weight=None, inv_freq=None, positions=None, offset=0, interleaved=False, eps=1e-6):
    """rotary_fwd of x / sqrt(mean(x^2) + eps) * weight, the mean over each head's features; without inv_freq the norm
    alone.  q_weight, k_weight: (dim), or None for ones; eps is a plain number."""
    return _head_fwd("norm fwd", True, q, k, q_weight, k_weight, inv_freq, positions, offset, interleaved, eps)


def norm_rotary_bwd(gq, gk, q, k, q_weight=None, k_weight=None, inv_freq=None, positions=None, offset=0, interleaved=False, eps=1e-6) -> HeadGrads:
    """Gradients of norm_rotary_fwd for upstream gradients gq and gk."""
    a, t = _head_plan("norm bwd", True, q, k, q_weight, k_weight, inv_freq, positions, offset, interleaved, eps, gq, gk)
    g = HeadGrads(_new(q), _new(k), _new(q_weight), _new(k_weight))
    ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=q.device)
    a.q, a.k, a.q_weight, a.k_weight = t[0].data_ptr(), _ptr(t[1]), _ptr(t[2]), _ptr(t[3])
    a.gq, a.gk, a.gx_q, a.gx_k = t[6].data_ptr(), _ptr(t[7]), g.q.data_ptr(), _ptr(g.k)
    a.gq_weight, a.gk_weight, a.workspace = _ptr(g.q_weight), _ptr(g.k_weight), ws.data_ptr()
    B_.call_with("fpde_head_rotary_bwd", a, q.device.index)
    return g


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, inv_freq, positions, offset, interleaved):
        ctx.save_for_backward(inv_freq, positions)
        ctx.how = (offset, interleaved)
        ctx.like = (q.shape, None if k is None else k.shape, q.dtype, q.device)
        ctx.set_materialize_grads(False)
        return rotary_fwd(q, k, inv_freq, positions, offset, interleaved)

    @staticmethod
    @once_differentiable
    def backward(ctx, gq, gk):
        inv_freq, positions = ctx.saved_tensors
        q_shape, k_shape, dt, dev = ctx.like
        if gq is None:
            gq = torch.zeros(q_shape, dtype=dt, device=dev)
        if gk is None and k_shape is not None:
            gk = torch.zeros(k_shape, dtype=dt, device=dev)
        return rotary_bwd(gq, gk, inv_freq, positions, *ctx.how) + (None, None, None, None)


class _NormRotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, inv_freq, positions, offset, interleaved, eps):
        ctx.save_for_backward(q, k, q_weight, k_weight, inv_freq, positions)
        ctx.how = (offset, interleaved, eps)
        ctx.set_materialize_grads(False)
        return norm_rotary_fwd(q, k, q_weight, k_weight, inv_freq, positions, offset, interleaved, eps)

    @staticmethod
    @once_differentiable
    def backward(ctx, gq, gk):
        q, k = ctx.saved_tensors[:2]
        gq = torch.zeros_like(q) if gq is None else gq
        gk = torch.zeros_like(k) if gk is None and k is not None else gk
        return tuple(norm_rotary_bwd(gq, gk, *ctx.saved_tensors, *ctx.how)) + (None,) * 5


def _no_gradient(name, t):
    if wants_grad(t):
        raise ValueError("%s has no gradient: detach it" % name)


def rotary(q, k, inv_freq, positions=None, offset=0, interleaved=False):
    """rotary_fwd, differentiable in q and k."""
    _no_gradient("inv_freq", inv_freq)
    return _Rotary.apply(q, k, inv_freq, positions, offset, interleaved)


def norm_rotary(q, k, q_weight=None, k_weight=None, inv_freq=None, positions=None, offset=0, interleaved=False, eps=1e-6):
    """norm_rotary_fwd, differentiable in q, k and the weights."""
    _no_gradient("inv_freq", inv_freq)
    return _NormRotary.apply(q, k, q_weight, k_weight, inv_freq, positions, offset, interleaved, eps)


# --------------------------------------------------------------------------------- linear attention
def _linear_args(q, k, v, log_decay, scale, state, step, go=None, gstate=None, backward=False):
    """As _conv_args, for linear attention."""
    _first("q", q, 3 if step else 4)
    dev, dt, batch, heads, dk = q.device, q.dtype, q.shape[0], q.shape[-2], q.shape[-1]
    if v.dim() != q.dim():
        raise ValueError("v has %d axes, expected %d" % (v.dim(), q.dim()))
    dv = v.shape[-1]
    a = B_.LinearArgs(dtype=B_.DTYPE_IDS[str(dt)], batch=batch, length=1 if step else q.shape[1], heads=heads, dk=dk, dv=dv, scale=scale)

    def view(name, t, like, width):
        t = _activation(name, t, like.shape[:-1] + (width,), dt, dev)
        setattr(a, name + "_batch", t.stride(0))
        setattr(a, name + "_node", 0 if step else t.stride(1))
        setattr(a, name + "_head", t.stride(-2))
        return t
    q, k, v = view("q", q, q, dk), view("k", k, q, dk), view("v", v, q, dv)
    log_decay = _dense("log_decay", log_decay, (heads,), torch.float32, dev)
    rest = (batch, heads, dk, dv)
    if step:
        _activation("state", state, rest, torch.float32, dev)
        if not state.is_contiguous():
            raise ValueError("state is updated in place and must be contiguous")
    else:
        state = _dense("state", state, rest, torch.float32, dev)
        if backward:
            go = view("go", go, q, dv)
            gstate = _dense("gstate", gstate, rest, torch.float32, dev)
        a.workspace_bytes = B_.lib().fpde_linear_attention_workspace_bytes(ctypes.byref(a), int(backward))
    return a, (q, k, v, log_decay, state, go, gstate)


def _linear_plan(kind, q, k, v, log_decay, scale, state, go=None, gstate=None):
    scale = _number("scale", scale)
    key = (kind, scale, _lay(q), _lay(k), _lay(v), _lay(log_decay), _lay(state), _lay(go), _lay(gstate))
    t = (q, k, v, log_decay, state, go, gstate)
    a = _plans.get(key)
    if a is None:
        a, taken = _linear_args(q, k, v, log_decay, scale, state, kind == "linear step", go, gstate, kind == "linear bwd")
        if _same(t, taken):
            _plans.keep(key, a)
        t = taken
    a.q, a.k, a.v, a.log_decay, a.state = t[0].data_ptr(), t[1].data_ptr(), t[2].data_ptr(), t[3].data_ptr(), _ptr(t[4])
    return a, t


def linear_attention_fwd(q, k, v, log_decay, scale=1.0, state=None):
    """For every row and head, with g = exp(log_decay[head]):

        S[t] = g S[t-1] + k[t] v[t]^T,  o[t] = scale * q[t] S[t],  S[-1] = state (batch, heads, dk, dv) or zeros

    q and k: (batch, length, heads, dk), v: (batch, length, heads, dv), up to 128 features each; log_decay: (heads); scale: a plain
    number.
    Returns (o (batch, length, heads, dv), the last state)."""
    return _linear_fwd(q, k, v, log_decay, scale, state, True)


def _linear_fwd(q, k, v, log_decay, scale, state, ends):
    """linear_attention_fwd; without `ends` no state leaves, which saves a third of the state's products in bf16."""
    a, t = _linear_plan("linear fwd", q, k, v, log_decay, scale, state)
    dev = q.device
    o, last = _new(v), None
    if ends:
        last = torch.empty((a.batch, a.heads, a.dk, a.dv), dtype=torch.float32, device=dev) if state is None else _new(state)
    a.o, a.state_out = o.data_ptr(), _ptr(last)
    if a.workspace_bytes:
        ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=dev)
        a.workspace = ws.data_ptr()
    B_.call_with("fpde_linear_attention_fwd", a, dev.index)
    return o, last


def linear_attention_bwd(go, q, k, v, log_decay, scale=1.0, state=None, gstate=None) -> LinearGrads:
    """Gradients of linear_attention_fwd for upstream gradients go of `o` and `gstate` of the last state."""
    return _linear_bwd(go, q, k, v, log_decay, scale, state, gstate, state is not None)


def _linear_bwd(go, q, k, v, log_decay, scale, state, gstate, of_state):
    a, t = _linear_plan("linear bwd", q, k, v, log_decay, scale, state, go, gstate)
    dev = q.device
    g = LinearGrads(_new(q), _new(k), _new(v), _new(state) if of_state else None)
    a.go, a.gstate_out = t[5].data_ptr(), _ptr(t[6])
    a.gq, a.gk, a.gv, a.gstate = g.q.data_ptr(), g.k.data_ptr(), g.v.data_ptr(), _ptr(g.state)
    if a.workspace_bytes:
        ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=dev)
        a.workspace = ws.data_ptr()
    B_.call_with("fpde_linear_attention_bwd", a, dev.index)
    return g


def linear_attention_step(state, q, k, v, log_decay, scale=1.0):
    """One node per row: q, k (batch, heads, dk), v (batch, heads, dv) -> o (batch, heads, dv); `state`
    (batch, heads, dk, dv) is moved on in place.  Not differentiable."""
    if torch.is_grad_enabled() and wants_grad(state, q, k, v, log_decay):
        return ValuesOnly.apply(linear_attention_step, state, q, k, v, log_decay, scale)
    a, t = _linear_plan("linear step", q, k, v, log_decay, scale, state)
    o = _new(v)
    a.state_out, a.o = state.data_ptr(), o.data_ptr()
    B_.call_with("fpde_linear_attention_step", a, q.device.index)
    _moved_on(state)
    return o


class _LinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, scale, state, ends):
        o, last = _linear_fwd(q, k, v, log_decay, scale, state, ends)
        ctx.save_for_backward(q, k, v, log_decay, state)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return o, last

    @staticmethod
    @once_differentiable
    def backward(ctx, go, glast):
        q, k, v, log_decay, state = ctx.saved_tensors
        if go is None:
            go = torch.zeros_like(v)
        g = _linear_bwd(go, q, k, v, log_decay, ctx.scale, state, glast, ctx.needs_input_grad[5])
        return g.q, g.k, g.v, None, None, g.state, None


def linear_attention(q, k, v, log_decay, scale=1.0, state=None, return_state=False):
    """linear_attention_fwd, differentiable in q, k, v and state; log_decay is a constant of the layer."""
    _no_gradient("log_decay", log_decay)
    o, last = _LinearAttention.apply(q, k, v, log_decay, scale, state, return_state)
    return (o, last) if return_state else o
