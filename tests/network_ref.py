"""Plain float64 implementations of the network operators on the CPU, and the
bounds that the GPU tests hold the kernels to.

Tolerances: a kernel's result is rounded once to its type (unit roundoff ``U``)
after arithmetic in float32 (or wider).  A float32 sum of k terms whose
magnitudes add up to m is off by at most about k * 2^-24 * m along its longest
chain of additions; ``close`` allows `chain` such roundings of `mag`.  Exponentials
and reciprocals are the hardware's, 1 ulp each, and count as two roundings."""
from __future__ import annotations

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def close(what, got, ref, chain, mag=None):
    """|got - ref| <= U |ref| + chain 2^-24 mag (mag: |ref| itself by default), element by element."""
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    g, r = got.detach().double().cpu(), ref.double().cpu()
    assert torch.equal(torch.isnan(g), torch.isnan(r)), f"{what}: NaN in other places"
    mag = r.abs() if mag is None else torch.as_tensor(mag, dtype=torch.float64).cpu()
    bound = U[got.dtype] * r.abs() + chain * 2.0 ** -24 * mag + TINY[got.dtype]
    off = torch.nan_to_num(g - r).abs() - torch.nan_to_num(bound, nan=float("inf"))
    if got.numel():
        worst = int(off.argmax())
        assert float(off.max()) <= 0, (f"{what}: {g.flatten()[worst]} for {r.flatten()[worst]}, allowed "
                                       f"{bound.expand_as(r).flatten()[worst]} at {worst} of {tuple(r.shape)}")


def randn(gen, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, dtype=torch.float64).to(dtype)


def d(t):
    return None if t is None else t.double().cpu()


def rms_norm(x, w, r, eps):
    s = x if r is None else x + r
    y = s * (s.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
    return (y if w is None else y * w), s


def rms_norm_bwd(dy, s, w, dsum, eps):
    """From the formula: ds = dsum + rho g - rho^3 mean(g s) s, dw = sum dy s rho."""
    rho = (s.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
    g = dy if w is None else dy * w
    ds = rho * g - rho ** 3 * (g * s).mean(-1, keepdim=True) * s
    dw = (dy * s * rho).flatten(0, -2).sum(0)
    return ds if dsum is None else ds + dsum, dw


def silu(p):
    return p * torch.sigmoid(p)


def causal_conv(x, w, b, act, state, lengths):
    """(y, state_out) from the definition, level by level."""
    B, L, D = x.shape
    W = w.shape[1]
    y = torch.zeros_like(x)
    last = torch.zeros(B, W - 1, D, dtype=x.dtype)
    for i in range(B):
        n = L if lengths is None else max(0, min(L, int(lengths[i])))
        h = torch.zeros(W - 1, D, dtype=x.dtype) if state is None else state[i]
        e = torch.cat((h, x[i, :n]))
        p = sum(w[:, k] * e[k:k + n] for k in range(W))
        if b is not None:
            p = p + b
        y[i, :n] = silu(p) if act else p
        last[i] = e[n:]
    return y, last


def softplus(x):
    return x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))


def selective_scan(u, delta, A, B, C, D, z, bias, sp, state, lengths):
    """(y, state after the last level) from the definition, level by level.  B, C: [b, L, G, N]."""
    Bn, L, Dn = u.shape
    group = torch.arange(Dn) // (Dn // B.shape[2])
    raw = delta if bias is None else delta + bias
    dt = softplus(raw) if sp else raw
    h = torch.zeros(Bn, *A.shape, dtype=u.dtype) if state is None else state
    n = torch.full((Bn,), L) if lengths is None else lengths.clamp(0, L)
    ys = []
    for t in range(L):
        on = (n > t)[:, None, None]
        new = torch.exp(dt[:, t, :, None] * A) * h + (dt[:, t] * u[:, t])[..., None] * B[:, t, group]
        h = torch.where(on, new, h)
        y = (h * C[:, t, group]).sum(-1)
        if D is not None:
            y = y + D * u[:, t]
        if z is not None:
            y = y * silu(z[:, t])
        ys.append(torch.where(on[..., 0], y, torch.zeros((), dtype=y.dtype)))
    return (torch.stack(ys, 1) if ys else torch.zeros_like(u)), h


def orthogonalize(g, steps, coeffs, eps):
    """Newton-Schulz from the definition, from the side that is smaller."""
    a, b, c = coeffs
    x = g / (g.norm() + eps)
    tall = g.shape[0] > g.shape[1]
    x = x.t() if tall else x
    for _ in range(steps):
        k = x @ x.t()
        x = a * x + (b * k + c * (k @ k)) @ x
    return x.t() if tall else x
