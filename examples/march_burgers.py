"""A network that marches u(x, t) along t, trained on the fused Burgers residual loss.

    python examples/march_burgers.py [--steps 200] [--nx 256] [--nt 128]

Each x node of the (x, t) grid is one row of `nt` nodes.  The network mixes a row with a causal
convolution and a selective state space scan (sequence.py); its output, with the initial and boundary
values built in, goes through the framework's residual loss (autograd.py), whose adjoint gives dL/du; the
projections are updated with orthogonalised momentum (optim.py), everything else with Adam.  At the end
the trained network is run one time node after the other, as a solver that does not know the whole
interval would run it, and has to give the same field.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_18020_b200 import optim, sequence  # noqa: E402
from paper_2607_18020_b200.autograd import fused_residual_loss  # noqa: E402

NU = 0.01 / math.pi


class Mixer(torch.nn.Module):
    """x + projection of (convolution -> scan, gated), all rows of the grid at once."""

    def __init__(self, width=64, states=16, taps=4):
        super().__init__()
        self.rank = max(1, width // 16)
        self.width, self.states = width, states
        self.norm = torch.nn.Parameter(torch.ones(width))
        self.into = torch.nn.Parameter(torch.randn(2 * width, width) / math.sqrt(width))
        self.taps = torch.nn.Parameter(torch.empty(width, taps).uniform_(-0.5, 0.5))
        self.taps_bias = torch.nn.Parameter(torch.zeros(width))
        self.select = torch.nn.Parameter(torch.randn(self.rank + 2 * states, width) / math.sqrt(width))
        self.rate = torch.nn.Parameter(torch.randn(width, self.rank) / math.sqrt(self.rank))
        step = torch.exp(torch.empty(width).uniform_(math.log(1e-2), math.log(0.3)))
        self.rate_bias = torch.nn.Parameter(torch.log(torch.expm1(step)))
        self.log_decay = torch.nn.Parameter(torch.log(torch.arange(1, states + 1, dtype=torch.float32)).repeat(width, 1))
        self.skip = torch.nn.Parameter(torch.ones(width))
        self.out = torch.nn.Parameter(torch.randn(width, width) / math.sqrt(width) * 0.5)

    def matrices(self):
        return [self.into, self.select, self.rate, self.out]

    def _split(self, v):
        bc = v @ self.select.t()
        return bc[..., :self.rank] @ self.rate.t(), bc[..., self.rank:self.rank + self.states], bc[..., self.rank + self.states:]

    def _rms(self, v):
        return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6) * self.norm

    def forward(self, v):
        """v: (rows, nodes, width)."""
        both = self._rms(v) @ self.into.t()
        a, z = both[..., :self.width], both[..., self.width:]
        a = sequence.causal_conv(a, self.taps, self.taps_bias)
        delta, b, c = self._split(a)
        y = sequence.selective_scan(a, delta, -torch.exp(self.log_decay), b, c, D=self.skip, z=z, delta_bias=self.rate_bias)
        return v + y @ self.out.t()

    def start(self, rows, device):
        return (torch.zeros(rows, self.taps.shape[1] - 1, self.width, device=device), torch.zeros(rows, self.width, self.states, device=device))

    def step(self, v, kept):
        """One node of every row: v (rows, width); `kept` (of start()) is moved on in place."""
        window, state = kept
        both = self._rms(v) @ self.into.t()
        a = sequence.causal_conv_step(both[:, :self.width], window, self.taps, self.taps_bias)
        delta, b, c = self._split(a)
        y = sequence.selective_scan_step(state, a, delta, -torch.exp(self.log_decay), b, c, D=self.skip, z=both[:, self.width:],
                                         delta_bias=self.rate_bias)
        return v + y @ self.out.t()


class March(torch.nn.Module):
    """u(x, t) = u0(x) + t (1 - x^2) net(x, u0, t): initial and boundary values hold for any weights."""

    def __init__(self, width=64, layers=2):
        super().__init__()
        self.embed = torch.nn.Linear(6, width)
        self.mixers = torch.nn.ModuleList(Mixer(width) for _ in range(layers))
        self.head = torch.nn.Linear(width, 1)
        torch.nn.init.zeros_(self.head.weight)
        torch.nn.init.zeros_(self.head.bias)

    def features(self, x, t):
        u0 = -torch.sin(math.pi * x)
        return u0, torch.stack(torch.broadcast_tensors(x, t, u0, torch.cos(math.pi * x), torch.sin(2 * math.pi * x), x * u0), -1)

    def forward(self, x, t):
        """x: (nx), t: (nt) -> (nx, nt)."""
        x, t = x[:, None], t[None, :]
        u0, f = self.features(x, t)
        v = self.embed(f)
        for m in self.mixers:
            v = m(v)
        return (u0 + t * (1 - x * x) * self.head(v)[..., 0]).contiguous()

    @torch.no_grad()
    def march(self, x, t):
        """The same field, one time node after the other."""
        kept = [m.start(x.shape[0], x.device) for m in self.mixers]
        nodes = []
        for k in range(t.shape[0]):
            u0, f = self.features(x, t[k])
            v = self.embed(f)
            for m, c in zip(self.mixers, kept):
                v = m.step(v, c)
            nodes.append(u0 + t[k] * (1 - x * x) * self.head(v)[:, 0])
        return torch.stack(nodes, 1)


def train(nx=256, nt=128, steps=200, width=64, seed=0, report=None):
    """Trains a March network; returns it with the losses and the grid's axes."""
    torch.manual_seed(seed)
    x, t = torch.linspace(-1, 1, nx, device="cuda"), torch.linspace(0, 1, nt, device="cuda")
    net = March(width).cuda()
    matrices = [p for m in net.mixers for p in m.matrices()]
    ids = {id(p) for p in matrices}
    muon = optim.Muon(matrices, lr=0.01)
    adam = torch.optim.Adam([p for p in net.parameters() if id(p) not in ids], lr=2e-3)
    spacing = (2.0 / (nx - 1), 1.0 / (nt - 1))
    losses = []
    for k in range(steps):
        loss = fused_residual_loss("burgers_1d_t", [net(x, t)], [], spacing, (NU,), ("one_sided", "one_sided"))
        muon.zero_grad(set_to_none=True)
        adam.zero_grad(set_to_none=True)
        loss.backward()
        muon.step()
        adam.step()
        losses.append(loss.detach())
        if report and (k % report == 0 or k == steps - 1):
            print("step %4d  residual loss %.4e" % (k, losses[-1].item()), flush=True)
    return net, [float(v) for v in losses], x, t


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--nx", type=int, default=256)
    ap.add_argument("--nt", type=int, default=128)
    a = ap.parse_args()
    net, losses, x, t = train(a.nx, a.nt, a.steps, report=20)
    with torch.no_grad():
        whole = net(x, t)
    node_by_node = net.march(x, t)
    print("one node after the other: largest difference %.2e" % (whole - node_by_node).abs().max().item())


if __name__ == "__main__":
    main()
