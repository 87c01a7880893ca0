"""Plain 64-bit forms of the sequence operators and of the orthogonalised update, on the CPU, one node
after the other, and the bounds their tests use.

Bounds (relative 2-norm of an output's error).  The kernels compute in fp32 and round once, so an output
of a 16-bit type may be off by its unit roundoff (2^-8 bf16 with its 8 bits,
2^-11 fp16 with its 11) plus the fp32 part; the fp32 part
gets the 1e-5 that every fp32 result of this library is held to."""
import torch

ROUND = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
FP32 = 1e-5
NS = (3.4445, -4.775, 2.0315)


def bound(dtype):
    return FP32 + ROUND[dtype]


def rel(a, b):
    a, b = a.detach().double().cpu(), b.detach().double().cpu()
    assert a.shape == b.shape, (a.shape, b.shape)
    if a.numel() == 0:
        return 0.0
    n = torch.linalg.vector_norm(b)
    d = torch.linalg.vector_norm(a - b)
    return float(d / n) if n > 0 else float(d)


def check(name, got, want, dtype=None):
    r = rel(got, want)
    lim = bound(dtype or got.dtype)
    assert r <= lim, "%s: relative error %.3e, bound %.3e" % (name, r, lim)


def d64(t):
    return None if t is None else t.detach().double().cpu()


def conv_ref(x, w, b, state, silu):
    """y and the window left, 64 bits, differentiable."""
    width = w.shape[1]
    if state is None:
        state = x.new_zeros(x.shape[0], width - 1, x.shape[2])
    full = torch.cat((state, x), 1)
    length = x.shape[1]
    pre = sum(full[:, j:j + length] * w[:, j] for j in range(width))
    if b is not None:
        pre = pre + b
    return (pre * torch.sigmoid(pre) if silu else pre), full[:, length:]


def scan_ref(u, delta, A, B, C, D, z, bias, softplus, state):
    """out and the last state, 64 bits, differentiable."""
    raw = delta if bias is None else delta + bias
    dt = torch.nn.functional.softplus(raw, threshold=100) if softplus else raw
    h = u.new_zeros(u.shape[0], u.shape[2], A.shape[1]) if state is None else state
    ys = []
    for t in range(u.shape[1]):
        h = torch.exp(dt[:, t, :, None] * A) * h + (dt[:, t] * u[:, t])[..., None] * B[:, t, None, :]
        ys.append((h * C[:, t, None, :]).sum(-1))
    y = torch.stack(ys, 1) if ys else torch.zeros_like(u)
    if D is not None:
        y = y + D * u
    return (y if z is None else y * z * torch.sigmoid(z)), h


def ortho_ref(g, steps, eps):
    x = g / (torch.linalg.vector_norm(g, dim=(-2, -1), keepdim=True) + eps)
    turned = x.shape[-2] > x.shape[-1]
    x = x.mT if turned else x
    for _ in range(steps):
        s = x @ x.mT
        x = NS[0] * x + (NS[1] * s + NS[2] * s @ s) @ x
    return x.mT if turned else x


class GuardedTorch:
    """Stands in for `torch` in a module under test: every tensor it gets from `empty` or `empty_like` has canaries on both
    sides and starts as NaN (so that what is not written shows)."""

    def __init__(self):
        self.all = []

    def __getattr__(self, name):
        return getattr(torch, name)

    def empty(self, *shape, dtype=torch.float32, device=None):
        shape = shape[0] if len(shape) == 1 and not isinstance(shape[0], int) else shape
        n = 1
        for k in shape:
            n *= int(k)
        e = torch.empty((), dtype=dtype).element_size()
        lead = 256
        raw = torch.full((lead + n * e + 256,), 0xA5, dtype=torch.uint8, device=device)
        body = raw[lead:lead + n * e]
        body.fill_(0xFF)                 # NaN in every floating type
        self.all.append((raw, lead, n * e))
        return body.view(dtype).view(*[int(k) for k in shape]) if n else torch.empty(*shape, dtype=dtype, device=device)

    def empty_like(self, t):
        return self.empty(t.shape, dtype=t.dtype, device=t.device)

    def check(self):
        for raw, lead, n in self.all:
            assert bool((raw[:lead] == 0xA5).all()) and bool((raw[lead + n:] == 0xA5).all()), "a guard band was overwritten"
