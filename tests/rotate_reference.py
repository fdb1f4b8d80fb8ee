"""Norm and rotation of heads, and their gradients, in 64 bits, with bounds of the kernels' roundings."""
import torch

HALF = 2.0 ** -8    # half a step of bf16, at most
SLACK = 2.0 ** -18  # fp32: the norm's factor, cosines and sines (2^-22 each) and a dozen operations; an angle of 2^31 positions is off by 2^31 2^-52 turns


def turned(x, pos, rot, pairs, base, back=False):
    """x [n][heads][dh], the dims of the pairs turned by the angles (or by their negatives)."""
    theta = pos.double()[:, None] * base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=x.device) / max(rot, 1))
    c, s = torch.cos(theta)[:, None], torch.sin(theta)[:, None] * (-1 if back else 1)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y = x.clone()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def sizes(x, rot, pairs):
    """For each dim how large what it is made of can be: |a| + |b| of its pair."""
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y = x.abs().clone()
    y[..., a], y[..., b] = x[..., a].abs() + x[..., b].abs(), x[..., a].abs() + x[..., b].abs()
    return y


def forward(x, pos, dh, w, eps, base, rot, pairs):
    v = x.double().view(x.shape[0], -1, dh)
    u = v / (v.square().mean(-1, keepdim=True) + eps).sqrt() * (1.0 if w is None else w.double())
    y = turned(u, pos, rot, pairs, base)
    return y.reshape(x.shape), (HALF * y.abs() + SLACK * sizes(u, rot, pairs)).reshape(x.shape)


def backward(x, dy, pos, dh, w, eps, base, rot, pairs):
    v, g = x.double().view(x.shape[0], -1, dh), dy.double().view(x.shape[0], -1, dh)
    r = 1.0 / (v.square().mean(-1, keepdim=True) + eps).sqrt()
    u, size = v * r, sizes(g, rot, pairs)
    g = turned(g, pos, rot, pairs, base, back=True)
    weight = torch.ones(dh, dtype=torch.float64, device=x.device) if w is None else w.double()
    dw, e_dw = (g * u).sum((0, 1)), 2 * SLACK * (size * u.abs()).sum((0, 1))
    gw = g * weight
    dx = r * (gw - u * (gw * u).mean(-1, keepdim=True))
    e = SLACK * r * (size * weight.abs() + u.abs() * (size * weight.abs() * u.abs()).mean(-1, keepdim=True))
    return {"dx": (dx.reshape(x.shape), (e + HALF * (dx.abs() + e)).reshape(x.shape)), "dw": (dw, e_dw)}
