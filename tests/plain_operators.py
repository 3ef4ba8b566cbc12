"""The operators around the step in 64 bits on the CPU, from their definitions (test infrastructure)."""
import math

import torch

D = 64


def turn(x, positions, base, interleaved, sign=1.0):
    """R(position) x for x [heads][tokens][64] (double), positions [tokens][axes]."""
    if positions is None:
        return x
    axes = positions.shape[1]
    w = D // axes
    y = x.clone()
    for ax in range(axes):
        for i in range(w // 2):
            a = sign * positions[:, ax].double() * float(base) ** (-2.0 * i / w)
            u = ax * w + (2 * i if interleaved else i)
            v = u + (1 if interleaved else w // 2)
            y[..., u] = x[..., u] * torch.cos(a) - x[..., v] * torch.sin(a)
            y[..., v] = x[..., v] * torch.cos(a) + x[..., u] * torch.sin(a)
    return y


def norm_rotate(x, w, b, norm, eps, positions, base, interleaved):
    """Differentiable; x, w, b double."""
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    if norm != "none":
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if w is not None:
        x = x * w
    if b is not None:
        x = x + b
    return turn(x, positions, base, interleaved)


def sees(n, m, causal):
    """[n][m]: query i, at key position i + m - n, sees key j."""
    if causal == 0:
        return torch.ones((n, m), dtype=torch.bool)
    pos = torch.arange(n) + m - n
    return (torch.arange(m)[None, :] // causal <= torch.floor(pos.double() / causal)[:, None]) & (pos >= 0)[:, None]


class Attention:
    """One head of one sequence: out, lse, gradients, and what the library's roundings can add up to.

    A result is rounded to bf16 once (2^-8 of itself), and so are P and dS where they enter a second product.  In front of that
    everything is fp32: a logit is 64 products added up and scaled, off by at most 2^-18 of scale * sum |q k| (64 roundings), P by
    that and the roundings of its exponent (2^-22 of |S| + |lse|), relative to itself.  The gradient takes out as the forward pass rounded it."""

    HALF = 2.0 ** -8

    def __init__(self, q, k, v, causal, scale, dout=None):
        q, k, v = q.double(), k.double(), v.double()
        n, m = q.shape[0], k.shape[0]
        see = sees(n, m, causal)
        S = (q @ k.t()) * scale
        S = torch.where(see, S, torch.full_like(S, -math.inf))
        lse = torch.logsumexp(S, 1) if m else torch.full((n,), -math.inf, dtype=torch.float64)
        some = see.any(1)
        P = torch.exp(S - torch.where(some, lse, torch.zeros_like(lse))[:, None])
        P = torch.where(see, P, torch.zeros_like(P))
        self.out, self.lse = P @ v, lse
        size = torch.where(see, (q.abs() @ k.abs().t()) * scale, torch.zeros_like(S)).amax(1) if m else torch.zeros(n, dtype=torch.float64)
        finite_lse = torch.where(some, lse, torch.zeros_like(lse)).abs()
        ep = 2.0 ** -17 * size + 2.0 ** -20 * (size + finite_lse) + 2.0 ** -20
        weight = P @ v.abs()
        self.out_tol = self.HALF * (weight + self.out.abs()) + 2 * ep[:, None] * weight
        self.lse_tol = ep + 2.0 ** -22 * finite_lse
        if dout is None:
            return
        d = dout.double()
        dP = d @ v.t()
        delta = (d * self.out).sum(1, keepdim=True)
        dS = P * (dP - delta)
        self.dq, self.dk, self.dv = (dS @ k) * scale, (dS.t() @ q) * scale, P.t() @ d
        delta_off = (d.abs() * self.out_tol).sum(1, keepdim=True)
        dS_off = P * (delta_off + 2.0 ** -17 * ((d.abs() @ v.abs().t()) + (d * self.out).abs().sum(1, keepdim=True)))
        dS_off = dS_off + (self.HALF + 2 * ep[:, None]) * (dS.abs() + dS_off)
        self.dq_tol = (dS_off @ k.abs()) * scale + self.HALF * self.dq.abs()
        self.dk_tol = (dS_off.t() @ q.abs()) * scale          # (the rounding of the sum over heads: the caller's)
        self.dv_tol = ((self.HALF + 2 * ep[:, None]) * P).t() @ d.abs()
