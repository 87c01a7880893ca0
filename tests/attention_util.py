"""Plain 64-bit forms of the rotation, the norm of heads and linear attention, on the CPU, the attention one node after
the other, and the bounds their tests use.

Bounds (relative 2-norm).  fp32 results are held to the 1e-5 that every fp32 result of this library is held to.  A 16-bit
result of the rotation or norm is rounded once: half a step, 2^-8 (bf16) or 2^-11 (fp16).  In the attention a factor of each
product may be rounded to 16 bits as well, which moves a sum by at most half a step of the sum of its terms' sizes; of terms of
random signs, as here, by half a step of the sum's own size in the 2-norm.  Together: two half steps."""
import torch
from seq_util import FP32, ROUND, rel


def attention_bound(dtype):
    return FP32 + 2 * ROUND[dtype]


def check_attention(name, got, want):
    r, lim = rel(got, want), attention_bound(got.dtype)
    assert r <= lim, "%s: relative error %.3e, bound %.3e" % (name, r, lim)


def rotary_ref(x, inv_freq, positions, offset, interleaved):
    n = inv_freq.shape[0]
    at = (torch.arange(x.shape[1])[None] if positions is None else positions) + offset
    angle = (at.double()[..., None] * inv_freq.double()).unsqueeze(2)
    c, s = torch.cos(angle), torch.sin(angle)
    if interleaved:
        a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        turned = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = x[..., :n], x[..., n:2 * n]
        turned = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((turned, x[..., 2 * n:]), -1)


def norm_ref(x, weight, eps):
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    return y if weight is None else y * weight


def linear_ref(q, k, v, log_decay, scale, state):
    """o and the last state, 64 bits, differentiable."""
    g = torch.exp(log_decay.double())[:, None, None]
    s = q.new_zeros(q.shape[0], q.shape[2], q.shape[3], v.shape[3]) if state is None else state
    out = []
    for t in range(q.shape[1]):
        s = g * s + k[:, t, :, :, None] * v[:, t, :, None, :]
        out.append(scale * (q[:, t, :, :, None] * s).sum(-2))
    return (torch.stack(out, 1) if out else 0.0 * v), s
