"""A network that marches in time, trained on the Burgers residual and answered
level by level.

    python examples/time_marching.py [--steps 200] [--nt 64] [--nx 128]

The network is a neural field generator for the space-time grid of
``workloads``' 1D+t Burgers operator: every node x is a sequence of time levels
and every level a row of features.  A block is

    y, s = RmsNorm(stream + branch)          root-mean-square norm, residual stream
    u, z = y W_in                            projections (plain products)
    u    = CausalConv(u)                     short convolution along time
    delta, B, C = u W_x, ...
    branch = SelectiveScan(u, delta, A, B, C, D, z) W_out

Its output is the field u(t, x).  The loss is the residual's (binding.ResidualLoss)
plus those of the initial and boundary values; matrices are updated by Muon,
everything else by Adam.  The trained network is then run as a rollout: one time
level at a time with the convolution's and the scan's carried states, which has to
give the window's field, and once more with the norm's output in 8 bits.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2607_18020_amd import binding as B  # noqa: E402
from paper_2607_18020_amd import network as N  # noqa: E402
from paper_2607_18020_amd import workloads as W  # noqa: E402


class Block(torch.nn.Module):
    def __init__(self, width, states, taps, gen):
        super().__init__()
        inner, rank = 2 * width, max(1, width // 16)
        self.inner, self.rank, self.states = inner, rank, states

        def matrix(rows, cols):
            return torch.nn.Parameter(torch.randn(rows, cols, generator=gen) / math.sqrt(rows))

        self.norm = torch.nn.Parameter(torch.ones(width))
        self.w_in = matrix(width, 2 * inner)
        self.conv_w = torch.nn.Parameter(torch.randn(inner, taps, generator=gen) / math.sqrt(taps))
        self.conv_b = torch.nn.Parameter(torch.zeros(inner))
        self.w_x = matrix(inner, rank + 2 * states)
        self.w_dt = matrix(rank, inner)
        # decay rates 1 .. states, step sizes of 0.01 to 0.2 of a level
        self.log_a = torch.nn.Parameter(torch.arange(1, states + 1).float().log().repeat(inner, 1))
        step = 0.01 * 20 ** torch.rand(inner, generator=gen)
        self.dt_bias = torch.nn.Parameter(torch.log(torch.expm1(step)))
        self.d = torch.nn.Parameter(torch.ones(inner))
        self.w_out = matrix(inner, width)

    def split(self, u):
        """delta, B and C of the convolved channels."""
        r, n = self.rank, self.states
        x = u @ self.w_x
        return x[..., :r] @ self.w_dt, x[..., r:r + n].contiguous(), x[..., r + n:].contiguous()

    def forward(self, branch, stream):
        """Whole windows [nodes, levels, width]; returns (branch, stream)."""
        y, stream = N.RmsNorm.apply(branch, stream, self.norm)
        u, z = (y @ self.w_in).split(self.inner, -1)
        u = N.CausalConv.apply(u, self.conv_w, self.conv_b)
        delta, b, c = self.split(u)
        y = N.SelectiveScan.apply(u, delta, -self.log_a.exp(), b, c, self.d, z, self.dt_bias)
        return y @ self.w_out, stream

    def state(self, nodes, device):
        return (torch.zeros(nodes, self.conv_w.shape[1] - 1, self.inner, device=device),
                torch.zeros(nodes, self.inner, self.states, device=device))

    def step(self, branch, stream, state, quant=None):
        """One level [nodes, width], the states updated in place."""
        if quant is None:
            y, stream = N.fpde_rms_norm(branch, self.norm, residual=stream)
        else:
            q, scales, stream = N.fpde_rms_norm(branch, self.norm, residual=stream, quant=quant)
            y = q.float() * scales.repeat_interleave(quant, 1)[:, :q.shape[1]] if quant else q.float() * scales
        u, z = (y @ self.w_in).split(self.inner, -1)
        u = N.fpde_causal_conv_step(u, state[0], self.conv_w, self.conv_b)
        delta, b, c = self.split(u)
        y = N.fpde_selective_step(state[1], u, delta, -self.log_a.exp(), b, c, D=self.d, z=z, delta_bias=self.dt_bias)
        return y @ self.w_out, stream


class TimeMarcher(torch.nn.Module):
    """u(t, x) from (t, x, u(0, x)): Fourier features, blocks, one output channel."""

    def __init__(self, width=64, blocks=2, states=16, taps=4, seed=0):
        super().__init__()
        gen = torch.Generator().manual_seed(seed)
        self.register_buffer("freq", torch.arange(1, 9).float() * math.pi)
        self.w_features = torch.nn.Parameter(torch.randn(2 * 16 + 3, width, generator=gen) / 6)
        self.blocks = torch.nn.ModuleList(Block(width, states, taps, gen) for _ in range(blocks))
        self.norm = torch.nn.Parameter(torch.ones(width))
        self.w_head = torch.nn.Parameter(torch.randn(width, 1, generator=gen) / math.sqrt(width))

    def features(self, t, x, u0):
        """[..., width] of every node's level; t, x, u0 broadcast."""
        t, x, u0 = torch.broadcast_tensors(t, x, u0)
        c = torch.stack((t, x), -1)[..., None] * self.freq
        f = torch.cat((c.sin().flatten(-2), c.cos().flatten(-2), torch.stack((t, x, u0), -1)), -1)
        return f @ self.w_features

    def forward(self, t, x, u0):
        """The field [levels, nodes] of a whole window."""
        branch = self.features(t[None, :], x[:, None], u0[:, None])
        stream = torch.zeros_like(branch)
        for b in self.blocks:
            branch, stream = b(branch, stream)
        y, _ = N.RmsNorm.apply(branch, stream, self.norm)
        return u0 + t[:, None] * (y @ self.w_head)[..., 0].t()

    @torch.no_grad()
    def rollout(self, t, x, u0, quant=None):
        """The same field, a level at a time."""
        states = [b.state(x.numel(), x.device) for b in self.blocks]
        out = torch.empty(t.numel(), x.numel(), device=x.device)
        for i in range(t.numel()):
            branch = self.features(t[i], x, u0)
            stream = torch.zeros_like(branch)
            for b, s in zip(self.blocks, states):
                branch, stream = b.step(branch, stream, s, quant)
            y, _ = N.fpde_rms_norm(branch, self.norm, residual=stream)
            out[i] = u0 + t[i] * (y @ self.w_head)[:, 0]
        return out


def problem(nt, nx, device):
    cfg = W.CONFIGS["burgers_1dt"]
    h = W.spacing("burgers_1dt", (nt, nx))
    t = torch.arange(nt, device=device) * h[0]
    x = -1 + torch.arange(nx, device=device) * h[1]
    return cfg, h, t.float(), x.float(), -torch.sin(math.pi * x).float()


def train(model, nt, nx, steps, device, lr=0.005, log=None):
    """Returns the losses of every step."""
    cfg, h, t, x, u0 = problem(nt, nx, device)
    matrices = [p for n, p in model.named_parameters() if p.dim() == 2 and "log_a" not in n and "conv" not in n]
    rest = [p for p in model.parameters() if all(p is not m for m in matrices)]
    optimisers = [N.Muon(matrices, lr=lr), torch.optim.Adam(rest, lr=lr)]
    losses = []
    for k in range(steps):
        u = model(t, x, u0)
        loss = B.ResidualLoss.apply(cfg.op, h, cfg.coeffs, [], u).float()
        loss = loss + (u[:, 0] ** 2).mean() + (u[:, -1] ** 2).mean()
        for o in optimisers:
            o.zero_grad()
        loss.backward()
        for o in optimisers:
            o.step()
        losses.append(loss.detach())
        if log and (k % log == 0 or k + 1 == steps):
            print(f"step {k:4d}  loss {loss.item():.4e}", flush=True)
    return torch.stack(losses)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--nt", type=int, default=64)
    ap.add_argument("--nx", type=int, default=128)
    ap.add_argument("--width", type=int, default=64)
    a = ap.parse_args()
    device = torch.device("cuda:0")
    model = TimeMarcher(a.width).to(device)
    train(model, a.nt, a.nx, a.steps, device, log=20)
    _, _, t, x, u0 = problem(a.nt, a.nx, device)
    with torch.no_grad():
        window = model(t, x, u0)
    for name, quant in (("rollout", None), ("rollout, norms in 8 bits", 128)):
        off = (model.rollout(t, x, u0, quant) - window).abs().max().item()
        print(f"{name}: at most {off:.2e} from the window's field of size {window.abs().max().item():.2f}")


if __name__ == "__main__":
    main()
