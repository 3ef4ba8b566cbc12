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
