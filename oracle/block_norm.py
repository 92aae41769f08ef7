"""Plain float64 oracle of the norm after a block, its gate and residual sum and the norm before the next block, and of its gradients (test
infrastructure only), written out from the definition.

    u = N_post(h) or h,  y = x_scale x + h_scale gate u,  n = N_pre(y) of y as it is stored
    t = dy + N_pre'(dn),  dx = x_scale t,  dgate = h_scale t u,  du = h_scale gate t,  dh = N_post'(du)
    N(z) = zhat w + b,  zhat = (z - mean) rstd;  N'(g) = rstd (a - mean(a) - zhat mean(a zhat)), a = g w (no mean for RMS)
"""
from __future__ import annotations

import torch


def statistics(z, kind, eps):
    """Mean and 1 / sqrt(var + eps) of every row; 0 where the kind ("none", "layer", "rms") has none."""
    zero = torch.zeros(z.shape[0], 1, dtype=torch.float64)
    if kind == "none":
        return zero, zero
    mean = z.mean(1, keepdim=True) if kind == "layer" else zero
    return mean, 1.0 / torch.sqrt(((z - mean) ** 2).mean(1, keepdim=True) + eps)


def norm(z, kind, eps, w, b):
    mean, rstd = statistics(z, kind, eps)
    out = (z - mean) * rstd * (1.0 if w is None else w)
    return out if b is None else out + b


def norm_gradient(g, z, kind, eps, w):
    """Gradients for z, w and b."""
    mean, rstd = statistics(z, kind, eps)
    zhat = (z - mean) * rstd
    a = g if w is None else g * w
    dz = a - zhat * (a * zhat).mean(1, keepdim=True)
    if kind == "layer":
        dz = dz - a.mean(1, keepdim=True)
    return rstd * dz, (g * zhat).sum(0), g.sum(0)


def forward(x, h, gate, post, pre, eps, x_scale, h_scale, w_post, b_post, w_pre, b_pre, stored=lambda y: y):
    u = h if post == "none" else norm(h, post, eps, w_post, b_post)
    y = h_scale * (u if gate is None else gate * u)
    if x is not None:
        y = y + x_scale * x
    s = stored(y)
    n = None if pre == "none" else norm(s, pre, eps, w_pre, b_pre)
    return y, n, torch.cat(statistics(h, post, eps) + statistics(s, pre, eps), 1)


def backward(dy, dn, h, y, gate, post, pre, eps, x_scale, h_scale, w_post, b_post, w_pre):
    """A dict of dx, dh, dgate (of every element), dw_post, db_post, dw_pre, db_pre."""
    out = {}
    t = torch.zeros_like(y) if dy is None else dy
    if pre != "none":
        dz, out["dw_pre"], out["db_pre"] = norm_gradient(dn, y, pre, eps, w_pre)
        t = t + dz
    out["dx"] = x_scale * t
    u = h if post == "none" else norm(h, post, eps, w_post, b_post)
    out["dgate"] = h_scale * t * u
    du = h_scale * t if gate is None else h_scale * gate * t
    out["dh"] = du
    if post != "none":
        out["dh"], out["dw_post"], out["db_post"] = norm_gradient(du, h, post, eps, w_post)
    return out
